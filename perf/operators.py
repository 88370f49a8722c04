"""The operators around a prompt's keys and values, as cases that can be timed and compared.

A program that serves a model with this library holds keys and values in pages until a prompt has been compressed, and
afterwards holds the kept rows and those of the tokens generated since.  Beside compressing, it makes three kinds of calls:

  * ``append``: new tokens' keys and values go into the pages of their sequences, keys and queries rotated by their
    positions on the way (``snapkv_append_paged``);
  * ``prompt``: causal attention over whole prompts packed one behind the other, with the rows' log-sum-exp, which the
    compression takes over (``snapkv_prompt_attention``);
  * ``decode``: attention of one new token per sequence over the paged cache (``snapkv_decode_attention_paged``).

Heads, head dims, page sizes and lengths are those of the repository's workloads and configurations; lengths of real
prompts are arbitrary, so most lengths here are odd.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GQA, MHA = {"Hq": 32, "Hkv": 8, "D": 128}, {"Hq": 32, "Hkv": 32, "D": 128}


def listed():
    return [
        # The tokens of one decoding step of eight users whose prompts were compressed: a row each, at a position far
        # beyond the row it is stored in.  Latency of a call.
        dict(GQA, name="append_step", kind="append", dtype="bf16", lengths="1,1,1,1,1,1,1,1", first=2048, last=2700,
             page=16, rot=128, interleaved=False, queries=True, keys_out=False, layout="fused", compressed=True),
        # Kept rows of four compressed prompts move into pages to be decoded from there: nothing is rotated again, the
        # rows lie head by head.
        dict(GQA, name="append_kept", kind="append", dtype="f16", lengths="2048,1024,2048,1024", first=0,
             last=0, page=32, rot=0, interleaved=False, queries=False, keys_out=False, layout="heads", compressed=False),
        # A multi-head layer's long prompts of one prefill, with the rotated keys left beside the pages as well for the
        # attention over the prompts.
        dict(MHA, name="append_large", kind="append", dtype="bf16", lengths="32749,4099,28471", first=0, last=0,
             page=16, rot=128, interleaved=False, queries=True, keys_out=True, layout="fused", compressed=False),
        # The shortest prompts there are: launches and latency.
        dict(GQA, name="prompt_short", kind="prompt", dtype="bf16", lengths="1,17,60", layout="fused"),
        # The prompts of one serving step, of very different lengths, in half precision.
        dict(GQA, name="prompt_batch", kind="prompt", dtype="f16", lengths="129,2100,700,64,1337,1025,333,1811",
             layout="fused"),
        # A multi-head layer with heads of 64, two prompts, tensors that lie head by head.
        dict(name="prompt_d64", kind="prompt", dtype="bf16", Hq=20, Hkv=20, D=64, lengths="5003,3001", layout="heads"),
        # A grouped-query layer's prompt of the library's 32K configuration, odd length.
        dict(GQA, name="prompt_32k", kind="prompt", dtype="bf16", lengths="32749", layout="fused"),
        # One GPU's share (one KV head and its four query heads) of a prompt of the long-context configuration.
        dict(name="prompt_131k", kind="prompt", dtype="bf16", Hq=4, Hkv=1, D=128, lengths="131071", layout="fused"),
        # One decoding step of one user over a short cache.  Latency of a step.
        dict(GQA, name="decode_one", kind="decode", dtype="bf16", lengths="2113", page=16),
        # A serving step of thirty-two users at very different lengths.
        dict(GQA, name="decode_batch", kind="decode", dtype="f16", page=16,
             lengths="1,16384,511,9001,130,12000,4097,777,15,2048,6001,300,10611,1500,64,8191,33,5000,1999,700,"
                     "14001,90,3333,260,7001,1024,17,13339,450,2900,8,11111"),
        # The step at batch 8 over uncompressed 16K prompts of a multi-head layer: what compression is compared with.
        dict(MHA, name="decode_mha", kind="decode", dtype="bf16",
             lengths="16384,16000,15999,16385,14000,16384,15001,16111", page=64),
        # One user at the long-context length: the split over the cache.
        dict(GQA, name="decode_long", kind="decode", dtype="bf16", lengths="131072", page=16),
    ]


def _lengths(case):
    return [int(n) for n in case["lengths"].split(",")]


def _text(lengths):
    return ",".join(map(str, lengths))


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = dict(rng.choice([GQA, GQA, MHA, {"Hq": 20, "Hkv": 20, "D": 64}, {"Hq": 32, "Hkv": 4, "D": 64},
                             {"Hq": 4, "Hkv": 1, "D": 128}, {"Hq": 6, "Hkv": 6, "D": 128}, {"Hq": 12, "Hkv": 4, "D": 128}]))
    kind = rng.choice(["append", "prompt", "prompt", "decode", "decode"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if kind == "append":
        step = rng.random() < 0.4
        if step:
            lengths = [1] * _log_uniform(rng, 1, 256)
        else:
            B, total = rng.randrange(1, 9), _log_uniform(rng, 8, 60000)
            lengths = [max(1, int(total * rng.uniform(0.1, 1.0) / B)) for _ in range(B)]
        moved = not step and rng.random() < 0.25
        D = heads["D"]
        return dict(heads, kind=kind, dtype=rng.choice([dtype, dtype, "f32"]) if sum(lengths) < 20000 else dtype,
                    lengths=_text(lengths), **({"first": 0, "last": 0} if rng.random() < 0.4 and not step else {"first": 1, "last": 4000}),
                    page=rng.choice([1, 8, 16, 16, 24, 32, 64, 128]), rot=0 if moved else rng.choice([D, D, D // 2]),
                    interleaved=not moved and rng.random() < 0.3, queries=not moved,
                    keys_out=not moved and not step and rng.random() < 0.5,
                    layout="heads" if moved else rng.choice(["fused", "tokens"]), compressed=step)
    if kind == "prompt":
        most = 8.0e12 if rng.random() < 0.5 else 2.0e11      # multiply-adds are bounded, not lengths alone
        longest = int(math.sqrt(most / (2.0 * heads["D"] * heads["Hq"])))
        if rng.random() < 0.4:
            lengths = [_log_uniform(rng, 1, min(longest, 131072))]
        else:
            B = rng.randrange(2, 17)
            cap = max(2, min(int(longest / math.sqrt(B)), 65536 // B))
            lengths = [_log_uniform(rng, 1, cap) for _ in range(B)]
        return dict(heads, kind=kind, dtype=dtype, lengths=_text(lengths), layout=rng.choice(["fused", "fused", "heads"]))
    # rows of all sequences and heads together stay below those of the largest listed step
    B = _log_uniform(rng, 1, 128)
    most = min(131072, int(120000 * 32 / (B * heads["Hkv"])))
    return dict(heads, kind=kind, dtype=dtype, page=rng.choice([8, 16, 16, 24, 32, 64, 128]),
                lengths=_text(_log_uniform(rng, 1, max(2, most)) for _ in range(B)))


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32)


def _rows(gen, T, heads, d, dtype, layout):
    """[T, heads, d] rows, stored token by token or (layout "heads") head by head."""
    if layout == "heads":
        return torch.empty((heads, T, d), device="cuda", dtype=dtype).normal_(generator=gen).transpose(0, 1)
    return torch.empty((T, heads, d), device="cuda", dtype=dtype).normal_(generator=gen)


def _projected(gen, case, T):
    """Queries, keys and values [T, heads, d]; layout "fused": columns of one tensor, as a projection leaves them.  N(0, 1),
    and the queries lean a little into what a few keys hold."""
    Hq, Hkv, d, dtype = case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    if case["layout"] == "fused":
        whole = torch.empty((T, (Hq + 2 * Hkv) * d), device="cuda", dtype=dtype).normal_(generator=gen)
        q, k, v = (t.view(T, -1, d) for t in whole.split([Hq * d, Hkv * d, Hkv * d], dim=1))
    else:
        q, k, v = (_rows(gen, T, h, d, dtype, case["layout"]) for h in (Hq, Hkv, Hkv))
    u = torch.randn((Hkv, d), generator=gen, device="cuda")
    u = (2.0 * u / u.norm(dim=-1, keepdim=True)).to(dtype)
    at = torch.randint(0, T, (1 + T // 64,), generator=gen, device="cuda").unique()
    k[at] = k[at] + u
    q.add_(u.repeat_interleave(Hq // Hkv, 0))
    return q, k, v


def _pool(gen, case, rows):
    """A pool of pages that other sequences use too, and the table of sequences of `rows` rows each."""
    page, dtype = case["page"], DTYPES[case["dtype"]]
    need = [-(-r // page) for r in rows]
    columns = max(1, max(need)) + 1
    pages = sum(need) + 3
    k = torch.empty((pages, page, case["Hkv"], case["D"]), device="cuda", dtype=dtype).normal_(generator=gen)
    v = torch.empty_like(k).normal_(generator=gen)
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((len(rows), columns), device="cuda", dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return k, v, table


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lengths, Hq, Hkv, d, dtype = _lengths(case), case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    B, T = len(lengths), sum(lengths)
    s = {"case": case}
    if case["kind"] == "decode":
        s["q"] = torch.empty((B, Hq, d), device="cuda", dtype=dtype).normal_(generator=gen)
        s["k_pages"], s["v_pages"], s["table"] = _pool(gen, case, lengths)
        s["lens"] = torch.tensor(lengths, device="cuda", dtype=torch.int32)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((B, Hq), device="cuda")
        s["longest"] = max(lengths)
        return s
    s["q"], s["k"], s["v"] = _projected(gen, case, T)
    s["cu"] = _offsets(lengths).cuda()
    if case["kind"] == "prompt":
        s["out"] = torch.empty((T, Hq, d), device="cuda", dtype=dtype)
        s["lse"] = torch.empty((Hq, T), device="cuda")
        return s
    starts = [random.Random(seed + b).randint(case["first"], case["last"]) for b in range(B)]
    s["starts"] = torch.tensor(starts, device="cuda", dtype=torch.int32)
    s["k_pages"], s["v_pages"], s["table"] = _pool(gen, case, [case["last"] + n for n in lengths])
    ahead = 29000 if case["compressed"] else 0       # a compressed prompt's next token is far beyond its row
    s["positions"] = torch.cat([torch.arange(a + ahead, a + ahead + n) for a, n in zip(starts, lengths)]).to(torch.int32).cuda()
    if case["rot"]:
        P, half = case["last"] + ahead + max(lengths), case["rot"] // 2
        angle = torch.arange(P, dtype=torch.float64, device="cuda")[:, None] * \
            10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    if not case["queries"]:
        del s["q"]
    else:
        s["q_out"] = torch.empty((T, Hq, d), device="cuda", dtype=dtype)
    if case["keys_out"]:
        s["k_out"] = torch.empty((T, Hkv, d), device="cuda", dtype=dtype)
    return s


def run(s):
    return {"append": _append, "prompt": _prompt, "decode": _decode}[s["case"]["kind"]](s)


def _append(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        snapkv.snapkv_append_paged(
            s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["starts"], cu_seqlens=s["cu"],
            positions=s["positions"] if c["rot"] else None, cos=s.get("cos"), sin=s.get("sin"),
            interleaved=c["interleaved"], q=s.get("q"), q_out=s.get("q_out"), k_out=s.get("k_out"))
        return {n: s[n] for n in ("k_pages", "v_pages", "q_out", "k_out") if n in s}
    T, page = s["k"].shape[0], c["page"]
    token = torch.arange(T, device="cuda", dtype=torch.int32)
    seq = torch.bucketize(token, s["cu"][1:], right=True)
    row = s["starts"][seq] + token - s["cu"][seq]
    slot = s["table"][seq, row // page].long() * page + row % page
    k, out = s["k"], {}
    if c["rot"]:
        at = s["positions"].long()
        cos, sin = s["cos"][at].unsqueeze(1), s["sin"][at].unsqueeze(1)
        k = _rotate(s["k"], cos, sin, c["interleaved"])
        if c["queries"]:
            out["q_out"] = _rotate(s["q"], cos, sin, c["interleaved"])
    for name, rows in (("k_pages", k), ("v_pages", s["v"])):
        s[name].view(-1, c["Hkv"], c["D"])[slot] = rows
        out[name] = s[name]
    if c["keys_out"]:
        out["k_out"] = k
    return {n: out[n] for n in ("k_pages", "v_pages", "q_out", "k_out") if n in out}


def _rotate(x, cos, sin, interleaved):
    half = cos.shape[-1]
    y = x.float()
    a, b = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if interleaved else (y[..., :half], y[..., half:2 * half])
    turned = (a * cos - b * sin, b * cos + a * sin)
    first = torch.stack(turned, dim=-1).flatten(-2) if interleaved else torch.cat(turned, dim=-1)
    return torch.cat([first, y[..., 2 * half:]], dim=-1).to(x.dtype)


def _prompt(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        snapkv.snapkv_prompt_attention(s["q"], s["k"], s["v"], s["cu"], s["out"], s["lse"])
        return s["out"], s["lse"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["D"]
    g = Hq // Hkv
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    begin = 0
    for L in _lengths(c):                                # the logits of a whole prompt need not fit: blocks of its rows
        block = max(1, min(L, (1 << 28) // (Hq * L)))
        kt = s["k"][begin:begin + L].float().permute(1, 2, 0).contiguous()
        v = s["v"][begin:begin + L].float().transpose(0, 1).contiguous()
        for r in range(0, L, block):
            e = min(r + block, L)
            q = s["q"][begin + r:begin + e].float().transpose(0, 1).reshape(Hkv, g * (e - r), d)
            x = torch.matmul(q, kt[:, :, :e].contiguous()).view(Hkv, g, e - r, e)
            x *= 1.0 / math.sqrt(d)
            x.masked_fill_(torch.arange(e, device="cuda") > torch.arange(r, e, device="cuda")[:, None], -math.inf)
            top = x.amax(dim=-1, keepdim=True)
            x = x.sub_(top).exp_()
            total = x.sum(dim=-1, keepdim=True)
            o = torch.matmul(x.view(Hkv, g * (e - r), e), v[:, :e].contiguous()).view(Hkv, g, e - r, d) / total
            out[begin + r:begin + e] = o.view(Hq, e - r, d).transpose(0, 1).to(out.dtype)
            lse[:, begin + r:begin + e] = (top + total.log()).view(Hq, e - r)
        begin += L
    return out, lse


def _decode(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        snapkv.snapkv_decode_attention_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"],
                                             s["longest"], s["out"], s["lse"])
        return s["out"], s["lse"]
    Hkv, d, page = c["Hkv"], c["D"], c["page"]
    B, Hq, _ = s["q"].shape
    columns = -(-s["longest"] // page)
    at = s["table"][:, :columns].long()
    kt = s["k_pages"][at].view(B, -1, Hkv, d).float().permute(0, 2, 3, 1).contiguous()
    x = torch.matmul(s["q"].float().view(B, Hkv, Hq // Hkv, d), kt) / math.sqrt(d)
    x.masked_fill_(torch.arange(columns * page, device="cuda") >= s["lens"].view(B, 1, 1, 1), -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    v = s["v_pages"][at].view(B, -1, Hkv, d).float().transpose(1, 2).contiguous()
    out = torch.matmul(x, v) / total
    return out.view(B, Hq, d).to(s["out"].dtype), (top + total.log()).view(B, Hq)


def exact(case, seed):
    s = prepare(case, seed)
    kind, Hkv, d = case["kind"], case["Hkv"], case["D"]
    g = case["Hq"] // Hkv
    if kind == "append":
        page, half, at = case["page"], case["rot"] // 2, 0
        new = {n: s[n].double() for n in ("q", "k") if n in s}
        if half:
            turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()].unsqueeze(1)
            for x in new.values():
                first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else \
                    (slice(0, half), slice(half, 2 * half))
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        table, starts = s["table"].tolist(), s["starts"].tolist()
        for b, n in enumerate(_lengths(case)):
            r = 0
            while r < n:
                column, line = divmod(starts[b] + r, page)
                m = min(n - r, page - line)
                k_pages[table[b][column], line:line + m] = new["k"][at + r:at + r + m]
                v_pages[table[b][column], line:line + m] = s["v"][at + r:at + r + m].double()
                r += m
            at += n
        out = {"k_pages": k_pages, "v_pages": v_pages}
        if case["queries"]:
            out["q_out"] = new["q"]
        if case["keys_out"]:
            out["k_out"] = new["k"]
        return out
    if kind == "prompt":
        out = torch.empty(s["out"].shape, device="cuda", dtype=torch.float64)
        lse = torch.empty(s["lse"].shape, device="cuda", dtype=torch.float64)
        at = 0
        for L in _lengths(case):
            step = max(1, min(L, (1 << 26) // L))
            for h in range(case["Hq"]):
                k, v = (s[n][at:at + L, h // g].double().contiguous() for n in ("k", "v"))
                for r in range(0, L, step):
                    e = min(r + step, L)
                    x = torch.mm(k[:e], (s["q"][at + r:at + e, h].double() / d ** 0.5).t().contiguous())   # keys x queries
                    x += torch.full((e, e - r), -math.inf, device="cuda", dtype=torch.float64).tril(-1 - r)
                    z = torch.logsumexp(x, dim=0)
                    out[at + r:at + e, h] = torch.mm(x.sub_(z).exp_().t().contiguous(), v[:e])
                    lse[h, at + r:at + e] = z
            at += L
        return out, lse
    out = torch.empty(s["out"].shape, device="cuda", dtype=torch.float64)
    lse = torch.empty(s["lse"].shape, device="cuda", dtype=torch.float64)
    table = s["table"].long()
    for b, S in enumerate(_lengths(case)):
        j = torch.arange(S, device="cuda")
        page, line = table[b, j // case["page"]], j % case["page"]
        for h in range(Hkv):
            x = torch.mm(s["k_pages"][page, line, h].double(), s["q"][b, h * g:(h + 1) * g].double().t().contiguous() / d ** 0.5)
            z = torch.logsumexp(x, dim=0)
            out[b, h * g:(h + 1) * g] = torch.mm((x - z).exp().t().contiguous(), s["v_pages"][page, line, h].double())
            lse[b, h * g:(h + 1) * g] = z
    return out, lse


def work(case):
    e, Hq, Hkv, d = DTYPES[case["dtype"]].itemsize, case["Hq"], case["Hkv"], case["D"]
    lengths = _lengths(case)
    B, T = len(lengths), sum(lengths)
    if case["kind"] == "append":
        # keys and values in and out once, queries and the second copy of the keys where asked for, a position's angles
        moved = 4 * Hkv + (2 * Hq if case["queries"] else 0) + (Hkv if case["keys_out"] else 0)
        turned = Hkv + (Hq if case["queries"] else 0)
        return {"bytes": T * (moved * d * e + 4 * case["rot"] + (4 if case["rot"] else 0)), "flops": 3 * T * turned * case["rot"]}
    if case["kind"] == "prompt":
        seen = sum(L * (L + 1) // 2 for L in lengths)
        return {"bytes": T * (2 * Hq + 2 * Hkv) * d * e + 4 * T * Hq, "flops": 4 * seen * Hq * d}
    return {"bytes": 2 * T * Hkv * d * e + B * Hq * (2 * d * e + 4) + sum(-(-S // case["page"]) for S in lengths) * 4,
            "flops": 4 * T * Hq * d}
