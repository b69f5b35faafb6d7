"""Performance cases of the paged key/value cache: what a serving program's attention layer asks of it.

Requests come and go, so their keys and values live in pages that a table lists for each of them, held in 16 bits or, for long
contexts, in 4 bits with a scale and a zero point for each of four interleaved groups of a row's channels.

  append  the newest tokens' rows of a packed query/key/value projection: queries and keys rotated, keys and values stored
          (``PagedKV.append``); pages in 4 bits are read back as the values they stand for (``PagedKV.read``);
  sdpa    attention of each sequence's newest tokens over its pages (``PagedKV.sdpa``): one token a sequence for a
          decode step, more for drafts and for a piece of a prompt.

Where ``own`` is false every operator is computed in its plain form.
"""
import math
import random

import numpy as np
import torch

own = False


def _case(kind, bits, seqs, tokens, heads, kv_heads, head_dim, length, page, dtype="f16", ragged=False, rope="", alibi=False,
          name=None):
    c = dict(kind=kind, bits=bits, seqs=seqs, tokens=tokens, heads=heads, kv_heads=kv_heads, head_dim=head_dim, length=length,
             page=page, dtype=dtype, ragged=ragged, rope=rope, alibi=alibi)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one token of one interactive request on a 7B layer
        _case("append", 16, 1, 1, 32, 32, 128, 1152, 16, rope="half", name="append_step_7b"),
        # four prompts of unequal, odd lengths, 256-wide heads
        _case("append", 16, 4, 1003, 16, 16, 256, 1003, 32, ragged=True, rope="interleaved", name="append_prompt_gptj"),
        # long prompts of a grouped-query model into 4 bits, and what the pages then hold
        _case("append", 4, 8, 2048, 32, 4, 128, 2048, 64, "bf16", ragged=True, rope="half", name="append4_prompt_gqa"),
        # the smallest use: a toy model's step
        _case("sdpa", 16, 1, 1, 4, 4, 64, 40, 16, name="sdpa_tiny"),
        # the interactive request again: latency
        _case("sdpa", 16, 1, 1, 32, 32, 128, 1152, 16, name="sdpa_llama2_7b"),
        # a serving batch of unequal lengths on 13B layers
        _case("sdpa", 16, 24, 1, 40, 40, 128, 1314, 16, ragged=True, name="sdpa_13b_ragged"),
        # few requests with long contexts, eight query heads to a kv head
        _case("sdpa", 16, 4, 1, 32, 4, 128, 65536, 64, "bf16", name="sdpa_gqa_long"),
        # many heads, ALiBi
        _case("sdpa", 16, 16, 1, 112, 112, 128, 1152, 32, "bf16", alibi=True, name="sdpa_bloom"),
        # the next piece of two long prompts
        _case("sdpa", 16, 2, 512, 32, 4, 128, 2560, 64, "bf16", name="sdpa_chunk"),
        # 256-wide heads in 4 bits
        _case("sdpa", 4, 16, 1, 16, 16, 256, 1152, 16, name="sdpa4_gptj"),
        # a large serving batch of unequal lengths, grouped-query, two draft tokens a request
        _case("sdpa", 4, 64, 2, 32, 4, 128, 8191, 32, "bf16", ragged=True, name="sdpa4_gqa_drafts"),
        # a batch of ordinary heads in 4 bits
        _case("sdpa", 4, 16, 1, 56, 56, 128, 2304, 64, name="sdpa4_opt"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    """One more case of the ranges above; no more bytes, operations and plain-form storage than the largest of them."""
    kind, bits = rng.choice(["append", "sdpa", "sdpa"]), rng.choice([16, 4])
    head_dim = rng.choice([64, 128, 128, 256])
    group = rng.choice([1, 1, 2, 4, 5, 8, 16])
    kv_heads = _log(rng, 1, 112 if group == 1 else 16)
    seqs, length = _log(rng, 1, 64), _log(rng, 1, 65536)
    if kind == "append":
        tokens = rng.choice([1, 1, 3, min(length, 2048), min(length, _log(rng, 2, 2048))])
    else:
        tokens = rng.choice([1, 1, 1, 1, 2, 5, _log(rng, 2, 512)])
    tokens = min(tokens, length)
    page, dtype = rng.choice([16, 32, 64, 128]), rng.choice(["f16", "bf16"])
    ragged = seqs > 1 and rng.random() < 0.6
    rope = rng.choice(["half", "interleaved", "half", ""]) if kind == "append" else ""
    alibi = kind == "sdpa" and rng.random() < 0.25
    while True:
        c = _case(kind, bits, seqs, min(tokens, length), kv_heads * group, kv_heads, head_dim, length, page, dtype, ragged, rope, alibi)
        values = seqs * length * kv_heads * head_dim                      # of K, and of V, with every sequence at full length
        scores = seqs * c["tokens"] * c["heads"] * length
        rows = seqs * c["tokens"] * (c["heads"] + 2 * kv_heads) * head_dim
        if values <= 2.6e8 and scores <= 9e7 and rows <= 9e7 and scores * head_dim * 4 <= 4.4e10:
            return c
        if seqs > 1 and (values > 2.6e8 or seqs >= 8):
            seqs = seqs * 2 // 3
            ragged = ragged and seqs > 1
        elif (scores > 9e7 or scores * head_dim * 4 > 4.4e10 or rows > 9e7) and tokens > 1:
            tokens = tokens * 2 // 3
        else:
            length = max(1, length * 2 // 3)


def _lens(case):
    """Each sequence's length after the call: the longest, or spread evenly between a quarter of it and the whole."""
    n, top = case["seqs"], case["length"]
    if not case["ragged"]:
        return [top] * n
    out = [max(1, int(top * (0.25 + 0.75 * ((b + 1) * 0.6180339887 % 1.0)))) for b in range(n)]
    out[n // 2] = top
    return out


def _new(case):
    """How many of them are new: for an append at most the sequence's length."""
    return [min(case["tokens"], x) for x in _lens(case)]


def work(case):
    n, T, H, Hkv, D = (case[k] for k in ("seqs", "tokens", "heads", "kv_heads", "head_dim"))
    lens = _lens(case)
    row = 2 * D if case["bits"] == 16 else D // 2 + 16                    # bytes of one key or value row in its page
    table = sum(-(-x // case["page"]) for x in lens) * 4
    if case["kind"] == "append":
        new = sum(_new(case))
        rotated = H * D * 2 * 2 if case["rope"] else 0
        angles = min(new, max(lens)) * D * 4 if case["rope"] else 0
        b = new * (2 * Hkv * (2 * D + row) + rotated) + angles
        if case["bits"] == 4:
            b += new * 2 * Hkv * (row + 2 * D)
        return {"bytes": float(b + n * 8), "flops": float(new * (H + Hkv) * D * 3)}
    seen = sum(sum(max(0, x - T + i + 1) for i in range(T)) for x in lens)
    return {"bytes": float(sum(lens) * 2 * Hkv * row + 2 * n * T * H * D * 2 + table + n * 4), "flops": 4.0 * D * H * seen}


# ---------------------------------------------------------------------------------------------------- pages in 4 bits
def _codes(x, dtype):
    """Codes 0..15, scales and zero points (in the pages' 16-bit type) of rows x [..., D]: channel d belongs to group d % 4."""
    g = x.float().unflatten(-1, (-1, 4))                                  # [..., D/4, 4]
    lo, hi = g.amin(-2, keepdim=True), g.amax(-2, keepdim=True)
    step = (hi - lo) / 15.0
    s, z = step.to(dtype), (lo + 8.0 * step).to(dtype)
    sf, zf = s.float(), z.float()
    c = torch.where(sf == 0, torch.full_like(g, 8.0), (torch.round((g - zf) / sf) + 8.0).clamp(0.0, 15.0))
    return c.flatten(-2).to(torch.uint8), s.squeeze(-2), z.squeeze(-2)


def _packed(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _parts(pages, case):
    """Views of 4-bit pages [pages, kv_heads, bytes]: codes [pages, kv_heads, page, D/2] and scales [.., page, 8], 16 bits."""
    ps, half = case["page"], case["head_dim"] // 2
    codes = pages[:, :, :ps * half].unflatten(-1, (ps, half))
    return codes, pages[:, :, ps * half:].view(_dtype(case)).unflatten(-1, (ps, 8))


def _values(codes, scales, kind):
    """What packed codes [..., D/2] and scales [..., 8] stand for."""
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(kind).unflatten(-1, (-1, 4)) - 8.0
    s, z = scales[..., :4].to(kind).unsqueeze(-2), scales[..., 4:].to(kind).unsqueeze(-2)
    return (c * s + z).flatten(-2)


def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _empty_pages(case, count, dev):
    ps, Hkv, D = case["page"], case["kv_heads"], case["head_dim"]
    if case["bits"] == 16:
        return torch.zeros(count, Hkv, ps, D, device=dev, dtype=_dtype(case))
    return torch.zeros(count, Hkv, ps * (D // 2 + 16), device=dev, dtype=torch.uint8)


class _State:
    pass


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = _dtype(case)
    n, T, H, Hkv, D, ps = (case[k] for k in ("seqs", "tokens", "heads", "kv_heads", "head_dim", "page"))
    s = _State()
    s.case = case
    lens = _lens(case)
    most = -(-max(lens) // ps)
    counts = [-(-x // ps) for x in lens]
    total = sum(counts) + 1
    # the sequences' pages lie all over the pool, as they do once requests have come and gone; entries past a sequence's end are -1
    at = np.random.default_rng(seed).permutation(total)
    table, used = np.full((n, most), -1, np.int32), 0
    for b, c in enumerate(counts):
        table[b, :c] = at[used:used + c]
        used += c
    s.table = torch.from_numpy(table).to(dev)
    s.lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    s.new = torch.tensor(_new(case), dtype=torch.int32, device=dev)
    s.slopes = None
    if case["alibi"]:
        s.slopes = torch.tensor([2.0 ** (-8.0 * (i + 1) / H) for i in range(H)], dtype=torch.float32, device=dev)
    s.k_pages, s.v_pages = _empty_pages(case, total, dev), _empty_pages(case, total, dev)
    if case["kind"] == "append":
        # a packed projection, as a fused QKV product leaves it
        x = torch.randn(n, T, H + 2 * Hkv, D, generator=g, device=dev, dtype=dt)
        s.q, s.k, s.v = x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]
        s.q_out = torch.zeros(n, T, H, D, device=dev, dtype=dt) if case["rope"] else None
        s.cos = s.sin = None
        if case["rope"]:
            i = torch.arange(D // 2, dtype=torch.float64, device=dev)
            angle = torch.arange(max(lens), dtype=torch.float64, device=dev)[:, None] * 10000.0 ** (-2.0 * i / D)
            s.cos, s.sin = torch.cos(angle).float(), torch.sin(angle).float()
        if case["bits"] == 4:
            s.k_out, s.v_out = (torch.zeros(n, T, Hkv, D, device=dev, dtype=dt) for _ in range(2))
        # which tokens of the padded batch there are, and where they go
        seq = [b for b, c in enumerate(_new(case)) for _ in range(c)]
        tok = [i for c in _new(case) for i in range(c)]
        s.seq, s.tok = torch.tensor(seq, device=dev), torch.tensor(tok, device=dev)
    else:
        s.q = torch.randn(n, T, H, D, generator=g, device=dev, dtype=dt)
        s.out = torch.zeros(n, T, H, D, device=dev, dtype=dt)
        for pages in (s.k_pages, s.v_pages):
            rows = torch.randn(total, Hkv, ps, D, generator=g, device=dev, dtype=dt)
            if case["bits"] == 16:
                pages.copy_(rows)
            else:
                codes, scales = _parts(pages, case)
                for lo in range(0, total, 4096):                          # (a part at a time: the steps between are in 32 bits)
                    c, a, z = _codes(rows[lo:lo + 4096], dt)
                    codes[lo:lo + 4096] = _packed(c)
                    scales[lo:lo + 4096] = torch.cat([a, z], -1)
            del rows
    if own:
        from paper_2401_05391_b200.pages import PagedKV
        s.h = PagedKV(H, Hkv, D, ps, total, dt, case["bits"], k_pages=s.k_pages, v_pages=s.v_pages)
    return s


# ------------------------------------------------------------------------------------------------------- the plain forms
def _turned(x, cos, sin, style):
    """Rows x [N, heads, D] turned by the angles of cos / sin [N, D/2]."""
    x, c, s = x.float(), cos[:, None], sin[:, None]
    if style == "half":
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def _plain_append(s):
    case = s.case
    dt = _dtype(case)
    pos = (s.lens - s.new).long()[s.seq] + s.tok
    page, off = s.table[s.seq, pos // case["page"]].long(), pos % case["page"]
    k, v = s.k[s.seq, s.tok], s.v[s.seq, s.tok]
    if case["rope"]:
        cos, sin = s.cos[pos], s.sin[pos]
        k = _turned(k, cos, sin, case["rope"]).to(dt)
        s.q_out[s.seq, s.tok] = _turned(s.q[s.seq, s.tok], cos, sin, case["rope"]).to(dt)
    if case["bits"] == 16:
        s.k_pages[page, :, off] = k
        s.v_pages[page, :, off] = v
        return [s.q_out, s.k_pages, s.v_pages]
    for x, pages, out in ((k, s.k_pages, s.k_out), (v, s.v_pages, s.v_out)):
        codes, scales = _parts(pages, case)
        c, a, z = _codes(x, dt)
        codes[page, :, off] = _packed(c)
        scales[page, :, off] = torch.cat([a, z], -1)
        out[s.seq, s.tok] = _values(codes[page, :, off], scales[page, :, off], torch.float32).to(dt)
    return [s.q_out, s.k_out, s.v_out]


def _gathered(pages, s):
    """[seqs, kv_heads, keys, D] in 32 bits: every sequence's rows, as many as the longest has pages for."""
    at = s.table.clamp(min=0).long()
    if s.case["bits"] == 16:
        x = pages[at].float()
    else:
        codes, scales = _parts(pages, s.case)
        x = _values(codes[at], scales[at], torch.float32)
    return x.transpose(1, 2).flatten(2, 3)


def _plain_sdpa(s):
    case = s.case
    n, T, H, Hkv, D = (case[k] for k in ("seqs", "tokens", "heads", "kv_heads", "head_dim"))
    G = H // Hkv
    q = s.q.float().view(n, T, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(n, Hkv, G * T, D)
    x = (torch.matmul(q, _gathered(s.k_pages, s).transpose(-1, -2)) / math.sqrt(D)).view(n, Hkv, G, T, -1)
    pos = s.lens[:, None] - T + torch.arange(T, device=q.device)                       # [seqs, tokens]
    away = torch.arange(x.shape[-1], device=q.device) - pos[..., None]                 # [seqs, tokens, keys]
    if s.slopes is not None:
        x = x + s.slopes.view(1, Hkv, G, 1, 1) * away[:, None, None].float()
    x = x.masked_fill((away > 0)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = x.sum(-1, keepdim=True)
    x = (x / torch.where(total == 0, torch.ones_like(total), total)).view(n, Hkv, G * T, -1)
    y = torch.matmul(x, _gathered(s.v_pages, s)).view(n, Hkv, G, T, D)
    return [y.permute(0, 3, 1, 2, 4).reshape(n, T, H, D).to(_dtype(case))]


def run(s):
    if not own:
        return _plain_append(s) if s.case["kind"] == "append" else _plain_sdpa(s)
    if s.case["kind"] == "sdpa":
        return [s.h.sdpa(s.q, s.table, s.lens, s.out, s.slopes)]
    if s.case["rope"]:
        s.h.append(s.k, s.v, s.table, s.lens, s.new, q=s.q, q_out=s.q_out, rope_cos=s.cos, rope_sin=s.sin, style=s.case["rope"])
    else:
        s.h.append(s.k, s.v, s.table, s.lens, s.new)
    if s.case["bits"] == 16:
        return [s.q_out, s.k_pages, s.v_pages]
    s.h.read(s.table, s.lens, s.case["tokens"], s.new, k=s.k_out, v=s.v_out)
    return [s.q_out, s.k_out, s.v_out]


# ------------------------------------------------------------------------------------------------------------ in 64 bits
def _exact_turn(x, pos, D, style, cos, sin):
    """The rotation as a complex product, in 64 bits, with the tables that the call is given."""
    w = torch.complex(cos[pos].double(), sin[pos].double())[:, None]                   # [tokens, 1, D/2]
    x = x.double()
    if style == "half":
        y = torch.complex(x[..., :D // 2], x[..., D // 2:]) * w
        return torch.cat([y.real, y.imag], -1)
    y = torch.view_as_complex(x.unflatten(-1, (D // 2, 2)).contiguous()) * w
    return torch.view_as_real(y).flatten(-2)


def _exact_held(x, dt):
    """What rows x hold in 4 bits: each group's range in 15 steps from the rounded scale and zero point."""
    x = x.to(dt).double()
    out = torch.empty_like(x)
    for j in range(4):
        y = x[..., j::4]
        lo, hi = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
        s = ((hi - lo) / 15).to(dt).double()
        z = (lo + (hi - lo) * 8 / 15).to(dt).double()
        c = torch.clamp(torch.round((y - z) / s) + 8, 0, 15)
        out[..., j::4] = torch.where(s > 0, z + (c - 8) * s, z.expand_as(y))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    n, T, H, Hkv, D, ps = (case[k] for k in ("seqs", "tokens", "heads", "kv_heads", "head_dim", "page"))
    lens, new, dt = _lens(case), _new(case), _dtype(case)
    if case["kind"] == "append":
        q_out = s.q_out.double() if case["rope"] else None
        ks, vs = (s.k_pages.double(), s.v_pages.double()) if case["bits"] == 16 else (s.k_out.double(), s.v_out.double())
        for b in range(n):
            m = new[b]
            pos = torch.arange(lens[b] - m, lens[b], device=s.lens.device)
            k, v = s.k[b, :m].double(), s.v[b, :m].double()
            if case["rope"]:
                k = _exact_turn(k, pos, D, case["rope"], s.cos, s.sin)
                q_out[b, :m] = _exact_turn(s.q[b, :m], pos, D, case["rope"], s.cos, s.sin)
            if case["bits"] == 4:
                ks[b, :m], vs[b, :m] = _exact_held(k, dt), _exact_held(v, dt)
            else:
                page, off = s.table[b][pos // ps].long(), pos % ps
                ks[page, :, off], vs[page, :, off] = k, v
        return [q_out, ks, vs]
    out = torch.zeros(n, T, H, D, dtype=torch.float64, device=s.q.device)
    for b in range(n):
        L = lens[b]
        at = s.table[b, :-(-L // ps)].long()
        kv = []
        for pages in (s.k_pages, s.v_pages):
            x = pages[at].double() if case["bits"] == 16 else None
            if x is None:
                codes, scales = _parts(pages, case)
                codes, scales = codes[at], scales[at].double()
                x = torch.empty(*codes.shape[:-1], D, dtype=torch.float64, device=out.device)
                for d4 in range(4):
                    c = (codes[..., d4 // 2::2] >> (4 * (d4 % 2))) & 15
                    x[..., d4::4] = (c.double() - 8) * scales[..., d4:d4 + 1] + scales[..., 4 + d4:5 + d4]
            kv.append(x.transpose(0, 1).reshape(Hkv, -1, D)[:, :L])
        for h in range(H):
            k, v = kv[0][h // (H // Hkv)], kv[1][h // (H // Hkv)]
            score = s.q[b, :, h].double() @ k.T / D ** 0.5                             # [tokens, keys]
            for_row = torch.arange(L, device=out.device)[None] - (L - T + torch.arange(T, device=out.device))[:, None]
            if s.slopes is not None:
                score = score + s.slopes[h].double() * for_row
            score = score.masked_fill(for_row > 0, -math.inf)
            p = torch.softmax(score, -1).nan_to_num(0.0)                               # (a row that sees nothing is zeros)
            out[b, :, h] = p @ v
    return [out]
