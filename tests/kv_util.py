"""The 4-bit cache and attention over it in 64 bits, one line per step of the definition; shares no code with the kernels."""
import math

import torch

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def power_of_two(e):
    """2^e in float64 for an integer tensor e (the exponent field itself: a device's pow need not be exact)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def hold(x):
    """Values [..., 32 n] (any float type) -> (codes, scale bytes, the values they stand for in float64): nearest grid value by
    search, ties to the even code; the smallest 2^e that brings a block's largest magnitude to at most 6, byte 2 .. 254."""
    b = x.double().unflatten(-1, (-1, 32))
    most = b.abs().amax(-1)
    byte = torch.full(most.shape, 2, dtype=torch.int64, device=x.device)
    for e in range(3, 255):
        byte = torch.where(most > 6.0 * 2.0 ** (e - 1 - 127), e, byte)
    bad = ~torch.isfinite(b).all(-1)
    unit = power_of_two(byte - 127)
    a = b.abs() / unit[..., None]
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    away = (a[..., None] - grid).abs()
    away = torch.where(torch.isnan(away), torch.inf, away)
    near = away.amin(-1, keepdim=True)
    code = torch.where(away == near, torch.tensor([0, 9, 2, 9, 4, 9, 6, 9], device=x.device), 9).amin(-1)   # the even one of a tie
    odd = (away == near).double().argmax(-1)
    code = torch.where(code == 9, odd, code)
    sign = torch.signbit(b)
    value = torch.where(sign, -grid[code], grid[code]) * unit[..., None]
    code = torch.where(bad[..., None], 0, code + 8 * sign)
    byte = torch.where(bad, 255, byte)
    value = torch.where(bad[..., None], torch.nan, value)
    return code.flatten(-2).to(torch.uint8), byte.to(torch.uint8), value.flatten(-2)


def pack(code):
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)


def values(codes, scales):
    """codes [..., dim / 2], scales [..., dim / 32] -> float64 [..., dim]"""
    grid = torch.tensor(GRID + [-g for g in GRID], dtype=torch.float64, device=codes.device)
    v = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], -1).flatten(-2)
    unit = torch.where(scales == 255, torch.nan, power_of_two(scales.long() - 127))
    return v * torch.repeat_interleave(unit, 32, -1)


def random_cache(gsi, n_pages, heads, dim, page, seed, device="cuda", poison=False):
    """A cache of random rows.  poison: scale bytes 255 everywhere until a row is written there."""
    g = torch.Generator(device=device).manual_seed(seed)
    u8 = dict(dtype=torch.uint8, device=device)
    codes = [torch.randint(0, 256, (n_pages, heads, page, dim // 2), generator=g, **u8) for _ in range(2)]
    scales = [torch.randint(124, 129, (n_pages, heads, dim // 32, page), generator=g, **u8) for _ in range(2)]
    if poison:
        scales = [torch.full_like(s, 255) for s in scales]
    return gsi.KvCache(codes[0], scales[0], codes[1], scales[1])


def keys_of(cache, pages, head, n):
    """K, V [n, dim] in float64 of the first n tokens of a list of page ids, and which of them lie on a page of the cache."""
    ids = torch.as_tensor(pages, device=cache.K.device).long()
    real = (ids >= 0) & (ids < cache.K.shape[0])
    ids = torch.where(real, ids, 0)
    k = values(cache.K[ids, head], cache.K_scale[ids, head].transpose(-1, -2)).reshape(-1, cache.dim)[:n]
    v = values(cache.V[ids, head], cache.V_scale[ids, head].transpose(-1, -2)).reshape(-1, cache.dim)[:n]
    return k, v, torch.repeat_interleave(real, cache.page)[:n]


def attention(cache, Q, q_start, kv_len, table, scale=None):
    """(O, lse, bound on |O error| for fp32 arithmetic, the same for bf16, bound on |lse error|), float64.

    The bounds, for a token whose largest |s| term sum is A = max_j scale sum_d |q_d k_jd| over the keys that it sees:
    each s is off by at most 2^-22 A (queries held to 2^-25 of a block's largest element, fp32 sums of up to 256 products with
    their roundings added in quadrature), its exponential by 2^-22 (1 + A) more (the product with log2 e and the maximum's
    subtraction round once each, the exponential to an ulp or two), and sums over keys and parts by 2^-21 relative.  An
    output is a weighted mean: with w_j off by delta relative, |O error| <= 2 delta sum_j w_j |v_j|.  bf16: a weight's rounding
    is 2^-9 relative, the output's 2^-9 of itself; both are taken twice.  Weights below 2^-126 of the largest, and what sums
    to that little, are no normal numbers in fp32: 2^-120 of the largest value per key comes on top of every bound."""
    T, heads, dim = Q.shape
    scale = dim ** -0.5 if scale is None else scale
    group = heads // cache.heads
    O = torch.zeros(Q.shape, dtype=torch.float64, device=Q.device)
    fine, coarse = torch.zeros_like(O), torch.zeros_like(O)
    lse = torch.full((T, heads), -math.inf, dtype=torch.float64, device=Q.device)
    off = torch.zeros_like(lse)
    start = list(range(T + 1)) if q_start is None else q_start.tolist()
    for b, n in enumerate(kv_len.tolist()):
        t0, t1 = start[b], start[b + 1]
        if t1 == t0 or n == 0:
            continue
        pages = table[b, :-(-n // cache.page)].tolist()
        for h in range(cache.heads):
            k, v, real = keys_of(cache, pages, h, n)
            q = Q[t0:t1, h * group:(h + 1) * group].double()
            s = scale * torch.einsum("tgd,kd->tgk", q, k)
            a = abs(scale) * torch.einsum("tgd,kd->tgk", q.abs(), k.abs())
            last = n - (t1 - t0) + torch.arange(t1 - t0, device=Q.device)
            seen = (torch.arange(n, device=Q.device)[None] <= last[:, None]) & real[None]
            some = seen.any(-1)[:, None]
            s = s.masked_fill(~seen[:, None], -math.inf)
            big = a.masked_fill(~seen[:, None], 0.0).amax(-1)
            top = torch.where(some, s.amax(-1), 0.0)
            p = torch.exp(s - top[..., None])
            p = torch.where(seen[:, None], p, 0.0)
            total = torch.where(some, p.sum(-1), 1.0)
            w = p / total[..., None]
            bad = torch.isnan(v)                                      # NaN reaches the tokens that see it, no others
            reached = torch.einsum("tk,kd->td", seen.double(), bad.double()) > 0
            held = torch.where(bad, 0.0, v)
            out = torch.where(reached[:, None], torch.nan, w @ held)
            O[t0:t1, h * group:(h + 1) * group] = out
            spread = w @ held.abs() + 2.0 ** -98 * n * held.abs().amax()      # 2^-120 once it is multiplied by delta, 2^-22 and more
            delta = 2.0 ** -22 * big + 2.0 ** -22 * (1 + big) + 2.0 ** -21
            fine[t0:t1, h * group:(h + 1) * group] = 2 * delta[..., None] * spread
            coarse[t0:t1, h * group:(h + 1) * group] = (2 * delta[..., None] + 2.0 ** -8) * spread + 2.0 ** -8 * out.abs()
            lse[t0:t1, h * group:(h + 1) * group] = torch.where(some, top + torch.log(total), -math.inf)
            off[t0:t1, h * group:(h + 1) * group] = torch.where(some, delta + 2.0 ** -22 * (top.abs() + torch.log(total).abs()), 0.0)
    return O, lse, fine, coarse, off


def check(got, got_lse, want, what=""):
    """got (and got_lse) against attention()'s answer: same NaN and infinities, the rest within its bounds."""
    O, lse, fine, coarse, off = want
    bound = coarse if got.dtype == torch.bfloat16 else fine
    g = got.double()
    assert torch.equal(torch.isnan(g), torch.isnan(O)), f"{what}: NaN in other places"
    err = torch.where(torch.isnan(O), 0.0, (g - O).abs())
    worst = (err / torch.where(bound > 0, bound, 1.0))
    assert bool((err <= torch.nan_to_num(bound, nan=0.0)).all()), f"{what}: error {float(err.max()):.3e}, {float(worst.max()):.2f} of its bound"
    if got_lse is not None:
        gl = got_lse.double()
        same = torch.isnan(gl) == torch.isnan(lse)
        assert bool(same.all()), f"{what}: NaN in other places of lse"
        inf = torch.isinf(lse)
        assert torch.equal(gl[inf], lse[inf]), f"{what}: lse of empty rows"
        e = torch.where(inf | torch.isnan(lse), 0.0, (gl - lse).abs())
        assert bool((e <= torch.nan_to_num(off, nan=0.0)).all()), f"{what}: lse error {float(e.max()):.3e}"
    return float(worst.max()) if worst.numel() else 0.0


def layout(gsi, lens, n_new, heads, kv_heads, dim, page, dtype, seed, poison=False, spare=3, width=None):
    """A cache whose requests hold `lens` tokens (their last n_new of this step), pages in random order, entries that nobody
    needs filled with ids that are no pages; rows written by the reference.  Returns cache, Q, q_start, kv_len, table."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare
    cache = random_cache(gsi, total, kv_heads, dim, page, seed + 1, poison=poison)
    width = max(1, max(need, default=0) + 1) if width is None else width
    table = torch.randint(-9, 0, (len(lens), width), generator=g, **i32)
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
        for j in range(n if poison else 0):
            pid = int(table[b, j])
            here = min(page, lens[b] - j * page)
            cache.K_scale[pid, :, :, :here] = torch.randint(124, 129, (kv_heads, dim // 32, here), generator=g, dtype=torch.uint8, device="cuda")
            cache.V_scale[pid, :, :, :here] = torch.randint(124, 129, (kv_heads, dim // 32, here), generator=g, dtype=torch.uint8, device="cuda")
    q_start = torch.zeros(len(lens) + 1, **i32)
    q_start[1:] = torch.cumsum(torch.tensor(n_new, **i32), 0)
    T = sum(n_new)
    Q = (torch.randn(T, heads, dim, generator=g, device="cuda") / 3).to(dtype)
    return cache, Q, q_start, torch.tensor(lens, **i32), table
