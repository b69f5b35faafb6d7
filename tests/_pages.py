"""The paged cache in plain tensor operations, for its tests: codes, rotation and attention, in 64 bits where values are compared."""
import math

import numpy as np
import torch


def codes_of(x, dtype):
    """(codes, scales, zero points) of rows x [..., D] of a 16-bit type, as the header gives them (fp32 steps)."""
    g = x.float().unflatten(-1, (-1, 4))
    lo, hi = g.amin(-2, keepdim=True), g.amax(-2, keepdim=True)
    step = (hi - lo) * torch.full((), 1.0 / 15.0, device=x.device)
    s, z = step.to(dtype), (lo + 8.0 * step).to(dtype)
    bad = ~torch.isfinite(g).all(-2, keepdim=True) | ~torch.isfinite(s) | ~torch.isfinite(z)
    s, z = s.masked_fill(bad, math.nan), z.masked_fill(bad, math.nan)
    c = (torch.round((g - z.float()) / s.float()) + 8.0).clamp(0.0, 15.0)
    c = torch.where((s.float() > 0) & ~bad, c, torch.full_like(c, 8.0))
    return c.flatten(-2).to(torch.uint8), s.squeeze(-2), z.squeeze(-2)


def split4(pages, page_size, head_dim, dtype):
    """Views of the codes [.., page, D/2] and the scales [.., page, 8] of 4-bit pages."""
    half = head_dim // 2
    return (pages[..., :page_size * half].unflatten(-1, (page_size, half)),
            pages[..., page_size * half:].view(dtype).unflatten(-1, (page_size, 8)))


def values4(codes, scales, kind=torch.float64):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).to(kind).unflatten(-1, (-1, 4)) - 8
    return (c * scales[..., None, :4].to(kind) + scales[..., None, 4:].to(kind)).flatten(-2)


def fill4(pages, rows, page_size, dtype):
    """Put rows [pages, kv_heads, page, D] into 4-bit pages."""
    codes, scales = split4(pages, page_size, rows.shape[-1], dtype)
    c, s, z = codes_of(rows, dtype)
    codes.copy_(c[..., 0::2] | (c[..., 1::2] << 4))
    scales.copy_(torch.cat([s, z], -1))


def turn(x, cos, sin, style):
    """Rows x [..., heads, D] by the angles of cos, sin [..., D/2], in the type of the tables."""
    x, c, s = x.to(cos.dtype), cos.unsqueeze(-2), sin.unsqueeze(-2)
    if style == "half":
        a, b = x.chunk(2, -1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    a, b = x[..., 0::2], x[..., 1::2]
    return torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)


def table_of(lens, page_size, pool, rng, entries=None, fill=-1):
    """A table whose sequences own pages from all over the pool."""
    counts = [-(-x // page_size) for x in lens]
    assert sum(counts) <= pool
    width = max([1] + counts) if entries is None else entries
    at, table, used = rng.permutation(pool), np.full((len(lens), width), fill, np.int32), 0
    for b, c in enumerate(counts):
        table[b, :c] = at[used:used + c]
        used += c
    return torch.from_numpy(table)


def sequence(cache, table, b, length):
    """(K, V, |parts of V|) [kv_heads, length, D] in 64 bits: what the rows of sequence b stand for, and the sizes that their sums are
    made of (4 bits: the code's and the zero point's part)."""
    at = table[b, :-(-length // cache.page_size)].long().to(cache.device)
    out = []
    for pages in (cache.k_pages, cache.v_pages):
        if cache.kv_bits == 16:
            x = pages[at].double()
            size, step = x.abs(), None
        else:
            codes, scales = split4(pages, cache.page_size, cache.head_dim, cache.dtype)
            codes, scales = codes[at], scales[at]
            x = values4(codes, scales)
            z = scales[..., None, 4:].double().expand(*x.shape[:-1], cache.head_dim // 4, 4).flatten(-2)
            size = (x - z).abs() + z.abs()
            step = scales[..., :4].double().abs().amax(-1, keepdim=True).expand_as(x)
        out.append([None if y is None else y.transpose(0, 1).flatten(1, 2)[:, :length] for y in (x, size, step)])
    return out


def attention(cache, q, table, lens, slopes=None, rounded=False):
    """(out, tolerance) in 64 bits, [n, q_len, heads, D].

    Tolerance of a kernel that holds scores, sums and accumulators in fp32 and rounds weights once and the output once to the dtype
    (u = half a step): u |out| for the output and u sum p |v| for the weights, v in the parts that are summed; a score's fp32
    error ds moves a weight by a factor e^ds, 2 ds sum p |v| at most with the sum it is divided by.  ds: D + 16 additions, each off by at most
    2^-22 of the terms' absolute sum (a tensor core cuts where fp32 would round); with 4-bit keys the terms are q (magic + code), up to 1040
    steps of the scale in fp16 and 144 in bf16.  ALiBi adds 2^-22 of its own size.  1e-5: exponentials, rescaling and the merge of splits.
    rounded: a kernel for many rows takes keys and values as the 16-bit numbers nearest to what 4-bit rows stand for: u |k| in the terms of a
    score, u |v| in those of the sum."""
    n, T, H, D = q.shape
    u = torch.finfo(cache.dtype).eps / 2
    G = H // cache.kv_heads
    out = torch.zeros(n, T, H, D, dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for b in range(n):
        L = int(lens[b])
        if L <= 0:
            continue
        (k, _, kstep), (v, size, _) = sequence(cache, table, b, L)
        pos = L - T + torch.arange(T, device=q.device)
        away = torch.arange(L, device=q.device)[None] - pos[:, None]                                   # [T, L]
        for h in range(H):
            qh = q[b, :, h].double()
            x = qh @ k[h // G].T / math.sqrt(D)
            terms = qh.abs() @ k[h // G].abs().T
            if kstep is not None:
                terms = terms + qh.abs().sum(-1, keepdim=True) * kstep[h // G][:, 0][None] * (1040.0 if cache.dtype == torch.float16 else 144.0)
            ds = (D + 16) * 2.0 ** -22 * terms / math.sqrt(D)
            if rounded:
                ds = ds + u * (qh.abs() @ k[h // G].abs().T) / math.sqrt(D)
            if slopes is not None:
                x = x + slopes[h].double() * away
                ds = ds + 2.0 ** -22 * (slopes[h].double() * away).abs()
            x = x.masked_fill(away > 0, -math.inf)
            p = torch.softmax(x, -1)
            p = torch.where(pos[:, None] < 0, torch.zeros_like(p), p)
            worst = torch.where(p > 0, ds, torch.zeros_like(ds))
            worst = (p * worst).sum(-1, keepdim=True) + worst * 1.0                                      # (of the sum, and of the weight)
            out[b, :, h] = p @ v[h // G]
            tol[b, :, h] = u * out[b, :, h].abs() + (p * ((2.05 if rounded else 1.05) * u + 1e-5 + 2 * worst.clamp(max=1.0))) @ size[h // G]
            tol[b, :, h] += L * 2.0 ** -30 * size[h // G].amax() + (2.0 ** -25 if cache.dtype == torch.float16 else 0.0)
    return out, tol


def check(got, out, tol):
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(out)), "finite where it should not be, or the other way round"
    err = torch.where(torch.isfinite(out), (got - out).abs(), torch.zeros_like(out))
    over = (err - tol).max().item()
    assert over <= 0, f"max error {err.max().item():.3e}, {over:.3e} over its bound"
