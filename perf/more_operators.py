"""Quantised paged caches and batches that share a prefix, as cases that can be timed and compared.

A server whose pages are full holds keys and values in 8 or 4 bits, and keeps one copy of what its users have in common.
Such a program makes four kinds of calls:

  * ``append``: new tokens' keys and values go into the pages as microscaled numbers, keys and queries rotated by their
    positions on the way (``snapkv_append_paged_mx``), and the rows just written are read back as the values that the cache
    now stands for (``snapkv_read_paged_mx``), which a prompt's next piece and the compression work on;
  * ``read``: rows of sequences leave the pages for contiguous storage (``snapkv_read_paged_mx``), as the compression takes
    a whole prompt;
  * ``decode``: attention of one new token per sequence over quantised pages (``snapkv_decode_attention_paged_mx``);
  * ``shared``: the same step for a batch whose sequences share long prefixes, each prefix read once for all that share
    it, and each sequence's own rows behind it (``snapkv_decode_attention_shared``).

A microscaled row holds its D values in blocks of 32: a power of two 2^e per block, held in one byte as e + 127, and 32
codes of 8 bits (e4m3) or 4 (e2m1, the even element in the low half of a byte).  e is the smallest with the block's
largest magnitude at most 2^e times the largest code's value (448 or 6), but not below -117; codes are the nearest
values, ties to even.  A block that holds an infinity or NaN has scale byte 255 and reads as NaN.

Heads, head dims, page sizes and lengths are those of the repository's workloads and configurations; lengths of real
prompts are arbitrary, so most lengths here are odd.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GQA, MHA = {"Hq": 32, "Hkv": 8, "D": 128}, {"Hq": 32, "Hkv": 32, "D": 128}
# of an element: smallest exponent of a normal number, bits behind the point, exponent of the largest, the largest over its power of two
ELEMENTS = {"fp8": (-6, 3, 8, 1.75), "fp4": (0, 1, 2, 1.5)}


def listed():
    return [
        # The tokens of one decoding step of eight users whose prompts were compressed, into an 8-bit cache: a row each, at a
        # position far beyond the row it is stored in.  Latency of two calls.
        dict(GQA, name="append_step", kind="append", cache="fp8", dtype="bf16", lengths="1,1,1,1,1,1,1,1", first=2048,
             last=2700, page=16, rot=128, interleaved=False, layout="fused", compressed=True),
        # Long prompts of one prefill of a multi-head layer into a 4-bit cache.
        dict(MHA, name="append_large", kind="append", cache="fp4", dtype="bf16", lengths="32749,4099,28471", first=0, last=0,
             page=16, rot=128, interleaved=False, layout="fused", compressed=False),
        # Kept rows of four compressed prompts leave a 4-bit cache, head by head.
        dict(GQA, name="read_kept", kind="read", cache="fp4", dtype="f16", lengths="2048,1024,2048,1024", first=0, last=0,
             page=32, layout="heads"),
        # A prompt of the 32K configuration leaves an 8-bit cache to be compressed: rows head by head, as the compression
        # takes them.
        dict(GQA, name="read_32k", kind="read", cache="fp8", dtype="bf16", lengths="32749", first=0, last=0, page=16,
             layout="heads"),
        # One decoding step of one user over a short cache.  Latency of a step.
        dict(GQA, name="decode_one", kind="decode", cache="fp8", dtype="bf16", lengths="2113", page=16),
        # A serving step of thirty-two users at very different lengths, in half precision.
        dict(GQA, name="decode_batch", kind="decode", cache="fp8", dtype="f16", page=16,
             lengths="1,16384,511,9001,130,12000,4097,777,15,2048,6001,300,10611,1500,64,8191,33,5000,1999,700,"
                     "14001,90,3333,260,7001,1024,17,13339,450,2900,8,11111"),
        # The step at batch 8 over uncompressed 16K prompts of a multi-head layer in 4 bits.
        dict(MHA, name="decode_mha", kind="decode", cache="fp4", dtype="bf16",
             lengths="16384,16000,15999,16385,14000,16384,15001,16111", page=64),
        # One user at the long-context length: the split over the cache.
        dict(GQA, name="decode_long", kind="decode", cache="fp4", dtype="bf16", lengths="131072", page=16),
        # Two answers to one compressed prompt, a few tokens in.  Latency of a step.
        dict(GQA, name="shared_two", kind="shared", cache="plain", dtype="bf16", prefixes="2048", groups="2", lengths="3,3",
             page=16),
        # Three documents with a few users each, of a model with heads of 64, in half precision.
        dict(name="shared_groups", kind="shared", cache="plain", dtype="f16", Hq=20, Hkv=20, D=64, prefixes="5003,9001,2100",
             groups="5,9,3", lengths="1,333,700,64,129,17,1025,2,450,90,300,15,33,511,260,1,130", page=16),
        # Sixty-four users of one long instruction.
        dict(GQA, name="shared_batch", kind="shared", cache="plain", dtype="bf16", prefixes="32749", groups="64",
             lengths=",".join(str(17 + 131 * i % 997) for i in range(64)), page=16),
        # Sixteen samples of an answer over a document of the long-context length held in 8 bits.
        dict(GQA, name="shared_131k", kind="shared", cache="fp8", dtype="bf16", prefixes="131071", groups="16",
             lengths=",".join(str(1 + 61 * i % 500) for i in range(16)), page=16),
    ]


def _ints(text):
    return [int(n) for n in text.split(",")]


def _text(lengths):
    return ",".join(map(str, lengths))


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads = dict(rng.choice([GQA, GQA, MHA, {"Hq": 20, "Hkv": 20, "D": 64}, {"Hq": 32, "Hkv": 4, "D": 64},
                             {"Hq": 4, "Hkv": 1, "D": 128}, {"Hq": 6, "Hkv": 6, "D": 128}, {"Hq": 12, "Hkv": 4, "D": 128}]))
    kind = rng.choice(["append", "read", "decode", "decode", "shared", "shared"])
    page, D = rng.choice([1, 8, 16, 16, 24, 32, 64, 128]), heads["D"]
    case = dict(heads, kind=kind, cache=rng.choice(["fp8", "fp4"]), dtype=rng.choice(["bf16", "bf16", "f16"]), page=page)
    if kind in ("append", "read"):
        step = kind == "append" and rng.random() < 0.4
        if step:
            lengths = [1] * _log_uniform(rng, 1, 256)
        else:
            B, total = rng.randrange(1, 9), _log_uniform(rng, 8, 60000)
            lengths = [max(1, int(total * rng.uniform(0.1, 1.0) / B)) for _ in range(B)]
        if sum(lengths) < 20000 and rng.random() < 0.25:
            case["dtype"] = "f32"
        case.update(lengths=_text(lengths), **({"first": 0, "last": 0} if rng.random() < 0.4 and not step else {"first": 1, "last": 4000}),
                    layout=rng.choice(["fused", "tokens", "heads"] if kind == "append" else ["heads", "heads", "tokens"]))
        if kind == "append":
            moved = not step and rng.random() < 0.25
            case.update(rot=0 if moved else rng.choice([D, D, D // 2]), interleaved=not moved and rng.random() < 0.3,
                        compressed=step)
        return case
    # rows of all sequences and heads together stay below those of the largest listed steps
    if kind == "decode":
        B = _log_uniform(rng, 1, 128)
        most = min(131072, int(120000 * 32 / (B * heads["Hkv"])))
        return dict(case, lengths=_text(_log_uniform(rng, 1, max(2, most)) for _ in range(B)))
    groups = [_log_uniform(rng, 1, 64) for _ in range(rng.choice([1, 1, 1, 2, 3, 5]))]
    G, B = len(groups), sum(groups)
    longest = min(131072, int(1.0e6 / (G * heads["Hkv"])), int(60.0e6 / (B * heads["Hq"])))
    return dict(case, cache=rng.choice(["plain", "plain", "fp8", "fp4"]), groups=_text(groups),
                prefixes=_text(_log_uniform(rng, 1, max(2, longest)) for _ in groups),
                lengths=_text(_log_uniform(rng, 1, max(2, min(1500, 300000 // (B * heads["Hkv"])))) for _ in range(B)))


def _offsets(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32)


def _rows(gen, T, heads, d, dtype, layout):
    """[T, heads, d] rows, stored token by token or (layout "heads") head by head."""
    if layout == "heads":
        return torch.empty((heads, T, d), device="cuda", dtype=dtype).normal_(generator=gen).transpose(0, 1)
    return torch.empty((T, heads, d), device="cuda", dtype=dtype).normal_(generator=gen)


def _projected(gen, case, T):
    """Queries, keys and values [T, heads, d]; layout "fused": columns of one tensor, as a projection leaves them."""
    Hq, Hkv, d, dtype = case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    if case["layout"] == "fused":
        whole = torch.empty((T, (Hq + 2 * Hkv) * d), device="cuda", dtype=dtype).normal_(generator=gen)
        q, k, v = (t.view(T, -1, d) for t in whole.split([Hq * d, Hkv * d, Hkv * d], dim=1))
    else:
        q, k, v = (_rows(gen, T, h, d, dtype, case["layout"]) for h in (Hq, Hkv, Hkv))
    k.mul_(_channels(gen, Hkv, d, dtype))
    return q, k, v


def _channels(gen, heads, d, dtype):
    """Keys have channels of very different size: a few are several times the others."""
    return torch.randn((heads, d), generator=gen, device="cuda").mul_(0.5).exp_().to(dtype)


def _table(gen, rows, page):
    """Pages enough for sequences of `rows` rows each and a few more, and the sequences' table of them."""
    need = [-(-r // page) for r in rows]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((len(rows), max(1, max(need)) + 1), device="cuda", dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return pages, table


def _pool(gen, case, pages):
    """The pages of keys and values: codes and scales, or rows of the case's type (no scales)."""
    page, H, d, dtype = case["page"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    scale, out = _channels(gen, H, d, torch.float32), {}
    for name in ("k", "v"):
        if case["cache"] == "plain":
            x = torch.empty((pages, page, H, d), device="cuda", dtype=dtype).normal_(generator=gen)
            out[name + "_pages"] = x.mul_(scale.to(dtype)) if name == "k" else x
            continue
        codes = torch.empty((pages, page, H, d if case["cache"] == "fp8" else d // 2), device="cuda", dtype=torch.uint8)
        scales = torch.empty((pages, page, H, d // 32), device="cuda", dtype=torch.uint8)
        step = max(1, (1 << 26) // (page * H * d))
        for p in range(0, pages, step):
            x = torch.randn((min(step, pages - p), page, H, d), generator=gen, device="cuda")
            codes[p:p + step], scales[p:p + step] = _encode(x * scale if name == "k" else x, case["cache"])
        out[name + "_pages"], out[name + "_scales"] = codes, scales
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lengths, Hq, Hkv, d, dtype = _ints(case["lengths"]), case["Hq"], case["Hkv"], case["D"], DTYPES[case["dtype"]]
    B, T, kind = len(lengths), sum(lengths), case["kind"]
    s = {"case": case}
    if kind in ("decode", "shared"):
        prefixes = _ints(case["prefixes"]) if kind == "shared" else []
        pages, table = _table(gen, prefixes + lengths, case["page"])
        s.update(_pool(gen, case, pages))
        s["q"] = torch.empty((B, Hq, d), device="cuda", dtype=dtype).normal_(generator=gen)
        s["table"], s["longest"] = table[len(prefixes):].contiguous(), max(lengths)
        s["lens"] = torch.tensor(lengths, device="cuda", dtype=torch.int32)
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((B, Hq), device="cuda")
        if prefixes:
            groups = _ints(case["groups"])
            s["prefix_table"], s["longest_prefix"] = table[:len(prefixes)].contiguous(), max(prefixes)
            s["prefix_lens"] = torch.tensor(prefixes, device="cuda", dtype=torch.int32)
            s["cu_groups"], s["most"] = _offsets(groups).cuda(), max(groups)
        return s
    starts = [random.Random(seed + b).randint(case["first"], case["last"]) for b in range(B)]
    s["starts"] = torch.tensor(starts, device="cuda", dtype=torch.int32)
    s["cu"] = _offsets(lengths).cuda()
    pages, s["table"] = _table(gen, [case["last"] + n for n in lengths], case["page"])
    s.update(_pool(gen, case, pages))
    for name in ("k_rows", "v_rows"):
        s[name] = _rows(gen, T, Hkv, d, dtype, "heads" if case["layout"] == "heads" else "tokens")
    if kind == "read":
        return s
    s["q"], s["k"], s["v"] = _projected(gen, case, T)
    ahead = 29000 if case["compressed"] else 0       # a compressed prompt's next token is far beyond its row
    s["positions"] = torch.cat([torch.arange(a + ahead, a + ahead + n) for a, n in zip(starts, lengths)]).to(torch.int32).cuda()
    if case["rot"]:
        P, half = case["last"] + ahead + max(lengths), case["rot"] // 2
        angle = torch.arange(P, dtype=torch.float64, device="cuda")[:, None] * \
            10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["q_out"] = torch.empty((T, Hq, d), device="cuda", dtype=dtype)
    else:
        del s["q"]
    return s


def run(s):
    return {"append": _append, "read": _read, "decode": _decode, "shared": _shared}[s["case"]["kind"]](s)


def _encode(x, cache):
    """Codes and scale bytes of rows [..., D] of float32 or float64: every step but the rounding to the grid is exact."""
    low, bits, top, most = ELEMENTS[cache]
    x = x.unflatten(-1, (-1, 32))
    large = x.abs().amax(dim=-1, keepdim=True)
    lost = ~(large < math.inf)                        # (infinity or NaN somewhere in the block)
    f, e = torch.frexp(torch.where(lost, 0.0, large))
    e = (e - 1 - top + (2.0 * f > most)).clamp_(min=-117)
    e = torch.where(large > 0, e, -117)
    y = torch.ldexp(torch.where(lost, 0.0, x), -e)
    own_e = torch.where(y == 0, low, torch.frexp(y.abs())[1] - 1).clamp_(min=low)
    m = torch.ldexp(y.abs(), bits - own_e).round_()   # (halves go to the even neighbour)
    code = ((own_e - low) * 2 ** bits + m).to(torch.uint8)
    code |= torch.signbit(y).to(torch.uint8) << (7 if cache == "fp8" else 3)
    code = code.flatten(-2)
    if cache == "fp4":
        code = code[..., 0::2] | code[..., 1::2] << 4
    return code, torch.where(lost, 255, e + 127).to(torch.uint8).squeeze(-1)


def _decoded(codes, scales, cache):
    """The values that codes and scale bytes stand for, in float32."""
    low, bits, _, _ = ELEMENTS[cache]
    if cache == "fp4":
        codes = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    sign = 1 << (7 if cache == "fp8" else 3)
    c = torch.arange(2 * sign, device="cuda")
    m, field = c % 2 ** bits, c % sign >> bits
    value = torch.where(field > 0, 2.0 ** bits + m, m.float()) * torch.exp2((field - 1).clamp(min=0).float() + low - bits)
    value = torch.where(c >= sign, -value, value)
    if cache == "fp8":
        value[127] = value[255] = math.nan
    unit = torch.ldexp(torch.ones(256, device="cuda"), torch.arange(256, device="cuda") - 127)
    unit[255] = math.nan
    return (value[codes.int()].unflatten(-1, (-1, 32)) * unit[scales.int()].unsqueeze(-1)).flatten(-2)


def _slots(s, T):
    """The row of the pool, pages laid out behind each other, that each of the packed tokens has."""
    token, page = torch.arange(T, device="cuda", dtype=torch.int32), s["case"]["page"]
    seq = torch.bucketize(token, s["cu"][1:], right=True)
    row = s["starts"][seq] + token - s["cu"][seq]
    return s["table"][seq, row // page].long() * page + row % page


def _pools(s):
    return s["k_pages"], s["k_scales"], s["v_pages"], s["v_scales"]


def _append(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        rot = bool(c["rot"])
        snapkv.snapkv_append_paged_mx(
            s["k"], s["v"], *_pools(s), s["table"], s["starts"], cu_seqlens=s["cu"],
            positions=s["positions"] if rot else None, cos=s.get("cos"), sin=s.get("sin"), interleaved=c["interleaved"],
            q=s.get("q"), q_out=s.get("q_out"))
        snapkv.snapkv_read_paged_mx(*_pools(s), s["table"], s["starts"], s["k_rows"], s["v_rows"], cu_seqlens=s["cu"])
        return {n: s[n] for n in ("q_out", "k_rows", "v_rows") if n in s}
    T, out, k = s["k"].shape[0], {}, s["k"].double()
    if c["rot"]:
        at = s["positions"].long()
        cos, sin = s["cos"][at].unsqueeze(1), s["sin"][at].unsqueeze(1)
        k = _rotate(k, cos.double(), sin.double(), c["interleaved"])       # (a code can be next to a border: 64 bits)
        out["q_out"] = _rotate(s["q"].float(), cos, sin, c["interleaved"]).to(s["q"].dtype)
    slot = _slots(s, T)
    for name, x in (("k", k), ("v", s["v"].float())):
        codes, scales = _encode(x, c["cache"])
        s[name + "_pages"].flatten(0, 1)[slot] = codes
        s[name + "_scales"].flatten(0, 1)[slot] = scales
    return {**out, **_read(s)}


def _read(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        snapkv.snapkv_read_paged_mx(*_pools(s), s["table"], s["starts"], s["k_rows"], s["v_rows"], cu_seqlens=s["cu"])
        return {n: s[n] for n in ("k_rows", "v_rows")}
    slot = _slots(s, s["k_rows"].shape[0])
    for name in ("k", "v"):
        x = _decoded(s[name + "_pages"].flatten(0, 1)[slot], s[name + "_scales"].flatten(0, 1)[slot], c["cache"])
        s[name + "_rows"].copy_(x)
    return {n: s[n] for n in ("k_rows", "v_rows")}


def _rotate(x, cos, sin, interleaved):
    half = cos.shape[-1]
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    turned = (a * cos - b * sin, b * cos + a * sin)
    first = torch.stack(turned, dim=-1).flatten(-2) if interleaved else torch.cat(turned, dim=-1)
    return torch.cat([first, x[..., 2 * half:]], dim=-1)


def _gathered(s, name, table, longest):
    """The first `longest` rows, up to a whole page, of the sequences of a table: [B, rows, Hkv, D] in float32."""
    c = s["case"]
    at = table[:, :-(-longest // c["page"])].long()
    x = s[name + "_pages"][at].flatten(1, 2)
    return x.float() if c["cache"] == "plain" else _decoded(x, s[name + "_scales"][at].flatten(1, 2), c["cache"])


def _logits(q, k, lens):
    """q [B, rows, Hkv, g, D] against k [B, keys, Hkv, D]: [B, Hkv, rows * g, keys], what lies behind lens masked."""
    x = torch.matmul(q.transpose(1, 2).flatten(2, 3), k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(q.shape[-1])
    return x.masked_fill_(torch.arange(k.shape[1], device="cuda") >= lens.view(-1, 1, 1, 1), -math.inf)


def _decode(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        snapkv.snapkv_decode_attention_paged_mx(s["q"], *_pools(s), s["table"], s["lens"], s["longest"], s["out"], s["lse"])
        return s["out"], s["lse"]
    B, Hq, d = s["q"].shape
    x = _logits(s["q"].float().view(B, 1, c["Hkv"], -1, d), _gathered(s, "k", s["table"], s["longest"]), s["lens"])
    top = x.amax(dim=-1, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(dim=-1, keepdim=True)
    v = _gathered(s, "v", s["table"], s["longest"]).transpose(1, 2).contiguous()
    out = torch.matmul(x, v) / total
    return out.view(B, Hq, d).to(s["out"].dtype), (top + total.log()).view(B, Hq)


def _shared(s):
    c = s["case"]
    if own:
        import paper_2404_14469_amd as snapkv
        snapkv.snapkv_decode_attention_shared(
            s["q"], s["k_pages"], s["v_pages"], s["prefix_table"], s["prefix_lens"], s["longest_prefix"], s["table"], s["lens"],
            s["longest"], s["out"], s["lse"], cu_groups=s["cu_groups"], k_scales=s.get("k_scales"), v_scales=s.get("v_scales"))
        return s["out"], s["lse"]
    B, Hq, d = s["q"].shape
    Hkv, most = c["Hkv"], s["most"]
    g, first = Hq // Hkv, s["cu_groups"].long()
    # the sequences of a group side by side, [G, most]: those of a smaller group are followed by others, which are not looked at
    member = (first[:-1, None] + torch.arange(most, device="cuda")).clamp_(max=B - 1)
    seq = torch.arange(B, device="cuda")
    group = torch.bucketize(seq, first[1:], right=True)
    place = seq - first[group]
    q = s["q"].float().view(B, Hkv, g, d)
    x = _logits(q[member], _gathered(s, "k", s["prefix_table"], s["longest_prefix"]), s["prefix_lens"])
    y = _logits(q.unsqueeze(1), _gathered(s, "k", s["table"], s["longest"]), s["lens"])
    shared = x.unflatten(2, (most, g)).amax(dim=-1)[group, :, place]          # [B, Hkv, g]
    top = torch.maximum(shared, y.amax(dim=-1))
    x = x.sub_(top[member].transpose(1, 2).reshape(len(member), Hkv, most * g, 1)).exp_()
    y = y.sub_(top.unsqueeze(-1)).exp_()
    total = x.sum(dim=-1).unflatten(2, (most, g))[group, :, place] + y.sum(dim=-1)
    out = torch.matmul(x, _gathered(s, "v", s["prefix_table"], s["longest_prefix"]).transpose(1, 2).contiguous())
    out = out.unflatten(2, (most, g))[group, :, place]
    out += torch.matmul(y, _gathered(s, "v", s["table"], s["longest"]).transpose(1, 2).contiguous())
    out /= total.unsqueeze(-1)
    return out.reshape(B, Hq, d).to(s["out"].dtype), (top + total.log()).view(B, Hq)


def _value(cache, codes, scales):
    """What codes [n, H, bytes] and scale bytes [n, H, blocks] stand for, in 64 bits, spelled out from the formats."""
    codes = codes.to(torch.int64)
    if cache == "fp4":
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
        nibbles = torch.empty(codes.shape[:-1] + (2 * codes.shape[-1],), dtype=torch.int64, device="cuda")
        nibbles[..., 0::2], nibbles[..., 1::2] = codes % 16, codes // 16
        x = grid[nibbles % 8] * (1 - 2 * (nibbles // 8))
    else:
        e, m = codes // 8 % 16, codes % 8
        x = torch.where(e == 0, m / 8.0 * 2.0 ** -6, (1 + m.double() / 8) * torch.pow(2.0, e.double() - 7))
        x = torch.where(codes % 128 == 127, math.nan, x) * (1 - 2 * (codes // 128))
    unit = torch.pow(2.0, scales.double() - 127)
    unit[scales == 255] = math.nan
    return x * unit.repeat_interleave(32, dim=-1)


def _nearest(x, cache):
    """Rows [n, H, D] in 64 bits as the cache's numbers: the nearest of the sorted grid, ties to the even code."""
    if cache == "fp4":
        grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        grid = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]
    grid = torch.tensor(grid, dtype=torch.float64, device="cuda")
    blocks = x.reshape(x.shape[0], x.shape[1], -1, 32)
    most = blocks.abs().amax(dim=-1, keepdim=True)
    unit = torch.full_like(most, 2.0 ** -117)
    for e in range(-116, 128):                       # the smallest power of two that holds the block
        unit = torch.where(most > grid[-1] * unit, 2.0 ** e, unit)
    y = blocks.abs() / unit
    above = torch.searchsorted(grid, y.contiguous()).clamp_(1, len(grid) - 1)
    below = above - 1
    up, down = grid[above] - y, y - grid[below]
    nearer = torch.where((up < down) | ((up == down) & (above % 2 == 0)), grid[above], grid[below])
    return (nearer * unit).copysign(blocks).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    kind, Hkv, d, cache, page = case["kind"], case["Hkv"], case["D"], case["cache"], case["page"]
    g, lengths = case["Hq"] // Hkv, _ints(case["lengths"])
    at = lambda row, a, n: (row[torch.arange(a, a + n, device="cuda") // page].long(), torch.arange(a, a + n, device="cuda") % page)
    if kind == "append":
        rows = {n: s[n].double() for n in ("q", "k", "v") if n in s}
        if case["rot"]:
            half = case["rot"] // 2
            turn = torch.complex(s["cos"].double(), s["sin"].double())[s["positions"].long()].unsqueeze(1)
            for x in (rows["q"], rows["k"]):
                first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else \
                    (slice(0, half), slice(half, 2 * half))
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
        out = {"q_out": rows["q"]} if case["rot"] else {}
        for n in ("k", "v"):
            out[n + "_rows"] = torch.cat([_nearest(x, cache) for x in rows[n].split(4096)])
        return out
    if kind == "read":
        out, starts = {}, s["starts"].tolist()
        for n in ("k", "v"):
            parts = []
            for b, m in enumerate(lengths):
                p, line = at(s["table"][b], starts[b], m)
                parts.append(_value(cache, s[n + "_pages"][p, line], s[n + "_scales"][p, line]))
            out[n + "_rows"] = torch.cat(parts)
        return out

    def held(n, row, m):                             # [m, Hkv, D]
        p, line = at(row, 0, m)
        x = s[n + "_pages"][p, line]
        return x.double() if cache == "plain" else _value(cache, x, s[n + "_scales"][p, line])

    out = torch.empty(s["out"].shape, device="cuda", dtype=torch.float64)
    lse = torch.empty(s["lse"].shape, device="cuda", dtype=torch.float64)
    prefixes, groups = ([0], [len(lengths)]) if kind == "decode" else (_ints(case["prefixes"]), _ints(case["groups"]))
    b = 0
    for i, (P, members) in enumerate(zip(prefixes, groups)):
        if P:
            kp, vp = (held(n, s["prefix_table"][i], P).transpose(0, 1).contiguous() for n in ("k", "v"))
        for b in range(b, b + members):
            k, v = (held(n, s["table"][b], lengths[b]) for n in ("k", "v"))
            for h in range(Hkv):
                q = s["q"][b, h * g:(h + 1) * g].double().t().contiguous() / d ** 0.5
                x = torch.mm(k[:, h].contiguous(), q)
                if P:
                    x = torch.cat([torch.mm(kp[h], q), x])
                z = torch.logsumexp(x, dim=0)
                w = (x - z).exp().t().contiguous()
                o = torch.mm(w[:, P:].contiguous(), v[:, h].contiguous())
                out[b, h * g:(h + 1) * g] = o + torch.mm(w[:, :P].contiguous(), vp[h]) if P else o
                lse[b, h * g:(h + 1) * g] = z
        b += 1
    return out, lse


def work(case):
    e, Hq, Hkv, d, cache = DTYPES[case["dtype"]].itemsize, case["Hq"], case["Hkv"], case["D"], case["cache"]
    row = d * e if cache == "plain" else (d if cache == "fp8" else d // 2) + d // 32      # bytes of a cached row
    lengths = _ints(case["lengths"])
    B, T, pages = len(lengths), sum(lengths), sum(-(-n // case["page"]) for n in lengths)
    if case["kind"] in ("append", "read"):
        moved = 2 * Hkv * (row + d * e)                                   # rows out of the pages
        if case["kind"] == "read":
            return {"bytes": T * moved + 4 * pages, "flops": T * 2 * Hkv * d}
        rot = case["rot"]
        moved += 2 * Hkv * (row + d * e) + ((2 * Hq * d * e + 4 * rot + 4) if rot else 0)
        # a rotation's products and sums, a quantised value's magnitude, scaling and rounding, and its way back
        return {"bytes": T * moved + 4 * pages, "flops": T * (3 * rot * (Hq + Hkv) + 8 * Hkv * d)}
    prefixes, groups = ([], []) if case["kind"] == "decode" else (_ints(case["prefixes"]), _ints(case["groups"]))
    seen = T + sum(P * n for P, n in zip(prefixes, groups))
    return {"bytes": 2 * (T + sum(prefixes)) * Hkv * row + B * Hq * (2 * d * e + 4)
            + 4 * (pages + sum(-(-P // case["page"]) for P in prefixes)), "flops": 4 * seen * Hq * d}
