"""What the tests of the steps around a paged cache share: inputs and the bounds on their outputs.

Bounds, from the kernels' arithmetic.  u = eps / 2 of the storage type (bf16 2^-8, fp16 2^-11, fp32 2^-24) is half a step
relative to a value, w = 2^-24 that of float32.

  rotation   two products and their sum in float32: at most 3 w (|a| + |b|) off before the one rounding to storage (cosine
             and sine are at most 1 in magnitude), so |got - want| <= u |want| + 4 w (|a| + |b|)
  logits     exact products, summed in float32 in some order: D w reach off, reach = sum_d |q_d k_d| / sqrt(D) at most; scaled
             and shifted by the running maximum with two more roundings at magnitude <= reach.  A probability relative to
             its row is thus off by d = 2 (D + 4) w reach + 2^-20 (the maximum moves with the logit; the exponential and the
             logarithm are good to 2^-21)
  sums       n terms in float32, in any order: n w
  output     a mean of v under probabilities that are rounded by at most c relative (prompts: c = u; one new token: two parts of
             the storage type, c = 2^-14 for bf16, 2^-20 for fp16), then rounded once:
             |got - want| <= u |want| + (c + 2 d + 2 n w) spread, spread = the mean of |v| under the same probabilities
             (fp16 probabilities are taken 2^7 times as large: those below 2^-14 / 2^7 of the largest are subnormal and lose up to half of
             2^-24, 2^-32 of it, each: n 2^-32 more)
  lse        d + n w + 2 w |lse|
"""
import numpy as np
import torch

W24 = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def num(t):
    return t.detach().double().cpu().numpy()


def check_attention(got, got_lse, want, want_lse, spread, reach, n, dtype, parts):
    """want, spread [..., D]; want_lse, reach [...] in the same order; n: rows that a query can see, at most."""
    D = want.shape[-1]
    u = half_step(dtype)
    c = {True: {torch.bfloat16: 2.0 ** -14, torch.float16: 2.0 ** -20}, False: {torch.bfloat16: u, torch.float16: u + n * 2.0 ** -32}}[parts][dtype]
    d = 2 * (D + 4) * W24 * reach + 2.0 ** -20
    bound = u * np.abs(want) + (c + 2 * d[..., None] + 2 * n * W24) * spread + 1e-30
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= bound).all(), (float((err / bound).max()), np.unravel_index((err / bound).argmax(), err.shape))
    if got_lse is not None:
        off = np.abs(got_lse - want_lse)
        lse_bound = d + n * W24 + 2 * W24 * np.abs(want_lse)
        assert (off <= lse_bound).all(), float((off / lse_bound).max())


def rows(gen, T, H, D, dtype, layout, scale=1.0):
    """[T, H, D] views of several storage orders, with what lies between the rows set to NaN."""
    if layout == "tokens":
        t = torch.empty((T, H, D), device="cuda", dtype=dtype)
    elif layout == "heads":
        t = torch.empty((H, T, D), device="cuda", dtype=dtype).transpose(0, 1)
    else:       # columns of a wider tensor, as a projection of queries, keys and values leaves them
        t = torch.full((T, (H + 2) * D), float("nan"), device="cuda", dtype=dtype)[:, D:-D].view(T, H, D)
    return t.copy_(scale * torch.randn((T, H, D), generator=gen, device="cuda"))


def seeded(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def offsets(lengths, first=0):
    return torch.tensor([first] + list(lengths)).cumsum(0).to(torch.int32).cuda()


def pool(gen, lens, page, Hkv, D, dtype, spare=3, fill=float("nan")):
    """Pages whose unowned rows hold `fill`, and a table in random order whose spare columns hold entries of no page."""
    need = [-(-max(0, n) // page) for n in lens]
    pages = sum(need) + spare
    k = torch.full((pages, page, Hkv, D), fill, device="cuda", dtype=dtype)
    v = k.clone()
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(1, max(need)) + 1), 1 << 30, device="cuda", dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return k, v, table


def fill_rows(gen, k, v, table, lens):
    page, Hkv, D = k.shape[1:]
    for b, n in enumerate(lens):
        j = torch.arange(max(0, n), device="cuda")
        slot = table[b, j // page].long() * page + j % page
        for t in (k, v):
            t.view(-1, Hkv, D)[slot] = torch.randn((max(0, n), Hkv, D), generator=gen, device="cuda").to(t.dtype)


def tables(P, half):
    a = torch.arange(P, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    return a.cos().float().cuda(), a.sin().float().cuda()
