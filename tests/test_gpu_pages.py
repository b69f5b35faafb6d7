"""The paged cache on a B200: store with rotation, attention over 16-bit and 4-bit pages, read-back, against plain forms in 64 bits."""
import math

import numpy as np
import pytest
import torch

import _pages as pg
from paper_2401_05391_b200 import segkv as sk
from paper_2401_05391_b200 import workloads as wl
from paper_2401_05391_b200.pages import PagedKV

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(*shape, dtype, g, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def filled(heads, kv_heads, D, ps, lens, dtype, bits, seed, scale=1.0, poison=False, spare=3):
    """A cache whose sequences of `lens` tokens hold random rows; `poison`: every row that no sequence owns is NaN or Inf."""
    g = gen(seed)
    pool = sum(-(-x // ps) for x in lens) + spare
    c = PagedKV(heads, kv_heads, D, ps, pool, dtype, bits)
    table = pg.table_of(lens, ps, pool, np.random.default_rng(seed))
    owned = torch.zeros(pool, ps, dtype=torch.bool)
    for b, x in enumerate(lens):
        for j in range(-(-x // ps)):
            owned[table[b, j], :min(ps, x - j * ps)] = True
    owned = owned.cuda()[:, None, :, None]
    for i, pages in enumerate((c.k_pages, c.v_pages)):
        rows = randn(pool, kv_heads, ps, D, dtype=dtype, g=g, scale=scale)
        if poison:
            rows = torch.where(owned, rows, torch.full_like(rows, math.inf if i else math.nan))
        if bits == 16:
            pages.copy_(rows)
        else:
            pg.fill4(pages, rows, ps, dtype)
    return c, table.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")


SHAPES = [
    # heads, kv_heads, D, page, q_len, lens
    (1, 1, 64, 16, 1, [1]),
    (4, 4, 64, 16, 1, [40, 1, 0, 17, 16]),
    (8, 2, 64, 64, 1, [300, 65, 64, 63]),
    (5, 1, 64, 32, 3, [2, 33, 257, 3]),
    (32, 2, 64, 16, 1, [700, 31]),
    (3, 3, 128, 16, 1, [1152, 15]),
    (16, 2, 128, 16, 1, [1, 129, 511, 0]),
    (20, 4, 128, 128, 2, [1000, 1, 128]),
    (16, 1, 128, 256, 1, [3000]),
    (14, 2, 128, 32, 1, [64, 65, 66, 127, 128, 129]),
    (6, 2, 128, 64, 40, [41, 39, 200]),
    (2, 2, 256, 16, 1, [257, 16, 1]),
    (8, 1, 256, 64, 1, [2048, 70]),
    (16, 1, 256, 32, 2, [100, 1, 0]),
]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:5])))
def test_attention(shape, dtype, bits):
    H, Hkv, D, ps, T, lens = shape
    seed = 7 * H + D + ps + T
    c, table, n_lens = filled(H, Hkv, D, ps, lens, dtype, bits, seed, poison=True)
    for alibi in (False, True):
        q = randn(len(lens), T, H, D, dtype=dtype, g=gen(seed + 1))
        slopes = wl.alibi_slopes(H).cuda() if alibi else None
        out = torch.full_like(q, math.nan)
        assert c.sdpa(q, table, n_lens, out, slopes) is out
        pg.check(out, *pg.attention(c, q, table, lens, slopes))
    assert c.get_error() == 0 and c.launch_count == 2
    c.destroy()


MANY = [
    # heads, kv_heads, D, page, q_len, lens: pieces of prompts, on the fifth-generation tensor cores where they fill them
    (1, 1, 64, 16, 128, [128]),
    (4, 4, 64, 16, 200, [200, 333, 150, 0, 1]),
    (32, 4, 128, 64, 64, [64, 65, 700, 63, 1]),
    (8, 8, 128, 16, 129, [129, 130, 256, 257, 100]),
    (12, 4, 128, 256, 150, [400, 151]),
    (16, 1, 128, 32, 300, [1000, 77]),
    (32, 1, 64, 128, 33, [33, 500]),
    (8, 2, 256, 16, 140, [140, 300, 17]),
    (2, 2, 256, 128, 257, [600]),
    (16, 16, 64, 32, 250, [250 + 7 * i for i in range(20)]),          # two groups of rows per CTA
    (8, 8, 128, 16, 256, [256 + 61 * (i % 5) for i in range(38)]),
]


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s[:5])))
def test_attention_of_many_rows(shape, dtype, bits):
    H, Hkv, D, ps, T, lens = shape
    seed = 7 * H + D + ps + T
    c, table, n_lens = filled(H, Hkv, D, ps, lens, dtype, bits, seed, poison=True)
    for alibi in (False, True):
        x = randn(len(lens), T, H + 2, D, dtype=dtype, g=gen(seed + 1))
        q = x[:, :, 1:H + 1] if D == 64 else x[:, :, :H].contiguous()
        slopes = wl.alibi_slopes(H).cuda() if alibi else None
        out = torch.full((len(lens), T, H, D), math.nan, dtype=dtype, device="cuda")
        c.sdpa(q, table, n_lens, out, slopes)
        pg.check(out, *pg.attention(c, q, table, lens, slopes, rounded=bits == 4))
        again = c.sdpa(q, table, n_lens, None, slopes)
        assert torch.equal(out, again)
    assert c.get_error() == 0
    c.destroy()


@pytest.mark.parametrize("bits,dtype,H,Hkv,D,T,lens", [
    (16, F16, 4, 1, 128, 1, [20011]), (4, F16, 2, 2, 128, 1, [3001, 64, 900]), (4, BF16, 1, 1, 256, 1, [8000]), (4, F16, 40, 40, 64, 1, [777] * 9),
    (16, F16, 3, 3, 128, 1, [200 + 37 * i for i in range(40)]), (16, BF16, 80, 80, 64, 1, [500, 0, 1300]), (4, F16, 4, 1, 128, 1, [20011]), (16, BF16, 16, 2, 64, 1, [9999, 3, 70]),
    (4, BF16, 16, 2, 256, 1, [5000, 12000]), (4, F16, 9, 1, 64, 2, [30001]), (16, F16, 2, 2, 256, 1, [7777]),
    (4, BF16, 8, 1, 128, 4, [4097] * 3), (16, F16, 32, 8, 128, 1, [200] * 64), (16, BF16, 24, 24, 64, 2, [13 * i for i in range(50)]),
    (16, F16, 40, 40, 128, 1, [70 * i for i in range(8)]), (16, F16, 16, 16, 256, 1, [250] * 19), (16, BF16, 8, 8, 128, 1, [1, 0] * 40)])
def test_work_groups_shared_by_many_ctas(bits, dtype, H, Hkv, D, T, lens):
    c, table, n_lens = filled(H, Hkv, D, 64, lens, dtype, bits, 900 + D)
    q = randn(len(lens), T, H, D, dtype=dtype, g=gen(901))
    out = c.sdpa(q, table, n_lens)
    pg.check(out, *pg.attention(c, q, table, lens))
    for _ in range(5):
        assert torch.equal(c.sdpa(q, table, n_lens), out)      # the order of the CTAs' arrival changes nothing
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("scale", [2.0 ** -12, 300.0])
def test_small_and_large_values(bits, scale):
    """Values whose scales would leave fp16 when multiplied into the weights; keys stay ordinary."""
    c, table, n_lens = filled(8, 2, 128, 16, [200, 77], F16, bits, 31)
    rows = randn(c.num_pages, 2, 16, 128, dtype=F16, g=gen(32), scale=scale)
    rows[0::3] *= 0.125
    if bits == 16:
        c.v_pages.copy_(rows)
    else:
        pg.fill4(c.v_pages, rows, 16, F16)
    q = randn(2, 1, 8, 128, dtype=F16, g=gen(33))
    pg.check(c.sdpa(q, table, n_lens), *pg.attention(c, q, table, [200, 77]))
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("heads,T", [(2, 1), (8, 1), (8, 5)])
@pytest.mark.parametrize("scale", [0.0, 1e-39, 1e-30, 1e30])
def test_queries_of_any_size_beside_a_bias(bits, heads, T, scale):
    """Queries so small that a key's distance, in their scores, would leave fp32; and so large that the bias is nothing."""
    lens = [200, 9]
    c, table, n_lens = filled(heads, 2, 128, 16, lens, BF16, bits, 34)
    q = randn(2, T, heads, 128, dtype=BF16, g=gen(35)) * scale
    for slopes in (wl.alibi_slopes(heads).cuda(), None):
        out, tol = pg.attention(c, q, table, lens, slopes)
        if scale > 1.0:                                       # (a score's error moves nothing where one key has all the weight)
            assert torch.isfinite(c.sdpa(q, table, n_lens, None, slopes)).all()
        else:
            pg.check(c.sdpa(q, table, n_lens, None, slopes), out, tol)
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scores_that_grow(bits, dtype):
    """Keys that turn towards the query along the sequence: the reference moves again and again; and one key that outweighs all."""
    D, L = 128, 700
    c, table, n_lens = filled(1, 1, D, 32, [L], dtype, bits, 41)
    q = randn(1, 1, 1, D, dtype=dtype, g=gen(42))
    rows = randn(c.num_pages, 1, 32, D, dtype=dtype, g=gen(43))
    order = table[0].long()
    ramp = torch.linspace(0, 8, order.numel() * 32, device="cuda").view(-1, 1, 32, 1)
    rows[order] = (rows[order].float() + ramp * q.float().view(1, 1, 1, D) / math.sqrt(D)).to(dtype)
    rows[order[3], 0, 5] = (q.view(D).float() * 3).to(dtype)
    if bits == 16:
        c.k_pages.copy_(rows)
    else:
        pg.fill4(c.k_pages, rows, 32, dtype)
    pg.check(c.sdpa(q, table, n_lens), *pg.attention(c, q, table, [L]))
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
def test_values_that_are_not_finite_stay_with_their_sequence(bits):
    lens = [50, 60, 70]
    c, table, n_lens = filled(4, 2, 64, 16, lens, F16, bits, 51)
    q = randn(3, 1, 4, 64, dtype=F16, g=gen(52))
    clean = c.sdpa(q, table, n_lens)
    page = int(table[1, 2])
    if bits == 16:
        c.v_pages[page, 0, 3] = math.inf
        c.k_pages[int(table[2, 0]), 1, 0, 0] = math.nan
    else:
        pg.split4(c.v_pages, 16, 64, F16)[1][page, 0, 3] = math.nan
        pg.split4(c.k_pages, 16, 64, F16)[1][int(table[2, 0]), 1, 0] = math.nan
    out = c.sdpa(q, table, n_lens)
    same = torch.ones(3, 4, dtype=torch.bool)
    same[1, :2] = False
    same[2, 2:] = False
    assert torch.equal(out[:, 0][same], clean[:, 0][same])
    assert not torch.isfinite(out[1, 0, :2]).any() and torch.isnan(out[2, 0, 2:]).all()
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("T,lens", [(3, [1, 2, 0, 7]), (200, [1, 130, 0, 450])])
def test_rows_that_see_nothing_are_zero_whatever_the_values_are(bits, T, lens):
    c, table, n_lens = filled(8, 2, 128, 16, lens, F16, bits, 53)
    if bits == 16:
        c.v_pages.fill_(math.nan)
        c.v_pages[..., ::3] = math.inf
    else:
        pg.split4(c.v_pages, 16, 128, F16)[1].fill_(math.nan)
    out = c.sdpa(randn(len(lens), T, 8, 128, dtype=F16, g=gen(54)), table, n_lens)
    for b, x in enumerate(lens):
        assert torch.equal(out[b, :max(T - x, 0)], torch.zeros_like(out[b, :max(T - x, 0)]))
        assert not torch.isfinite(out[b, max(T - x, 0):]).any()
    c.destroy()


@pytest.mark.parametrize("heads,T", [(2, 1), (8, 1), (8, 3)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_group_that_is_not_held_leaves_the_others_as_they_are(dtype, heads, T):
    c, table, n_lens = filled(heads, 2, 128, 16, [60, 200], dtype, 4, 55)
    q = randn(2, T, heads, 128, dtype=dtype, g=gen(56))
    clean = c.sdpa(q, table, n_lens)
    scales = pg.split4(c.v_pages, 16, 128, dtype)[1]
    for page in (int(table[0, 1]), int(table[1, 7])):
        scales[page, :, 5, 2] = math.nan                       # scale and zero point of group 2
        scales[page, :, 5, 6] = math.nan
    out = c.sdpa(q, table, n_lens)
    for group in range(4):
        if group == 2:
            assert torch.isnan(out[..., group::4]).all()
        else:
            assert torch.equal(out[..., group::4], clean[..., group::4])
    c.destroy()


def test_query_rows_of_a_packed_projection():
    c, table, n_lens = filled(8, 2, 64, 16, [33, 90], F16, 16, 61)
    x = randn(2, 3, 8 + 4, 64, dtype=F16, g=gen(62))
    assert torch.equal(c.sdpa(x[:, :, :8], table, n_lens), c.sdpa(x[:, :, :8].contiguous(), table, n_lens))
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
def test_offsets_beyond_32_bits(bits):
    """A pool of more than 2^32 bytes whose last pages are used."""
    D, Hkv, ps = 128, 8, 256
    per = Hkv * ps * (2 * D if bits == 16 else D // 2 + 16)
    pool = 2 ** 32 // per + 40
    c = PagedKV(8, Hkv, D, ps, pool, F16, bits)
    lens = [ps * 3 + 5, 9]
    table = torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    table[0] = torch.tensor([pool - 1, pool - 9, 0, pool - 2])
    table[1, 0] = pool - 30
    n_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    k, v = (randn(2, max(lens), Hkv, D, dtype=F16, g=gen(70 + i)) for i in range(2))
    c.append(k, v, table, n_lens, n_lens)
    rk, rv = c.read(table, n_lens, max(lens), n_lens)
    for b, L in enumerate(lens):
        if bits == 16:
            assert torch.equal(rk[b, :L], k[b, :L]) and torch.equal(rv[b, :L], v[b, :L])
        assert not rk[b, L:].any() and not rv[b, L:].any()
    q = randn(2, 1, 8, D, dtype=F16, g=gen(73))
    pg.check(c.sdpa(q, table, n_lens), *pg.attention(c, q, table, lens))
    assert c.get_error() == 0
    c.destroy()


# ------------------------------------------------------------------------------------------------------------- the store
APPENDS = [
    # heads, kv_heads, D, page, tokens, lens, new
    (4, 4, 64, 16, 1, [1, 40, 17, 0, 16], None),
    (6, 2, 128, 32, 1, [100], None),
    (5, 1, 256, 64, 3, [2, 3, 70], None),
    (8, 8, 128, 16, 50, [50, 49, 1, 77], [50, 20, 1, 33]),
    (3, 3, 64, 128, 257, [300, 257, 20], [257, 0, 20]),
    (4, 2, 256, 16, 33, [33, 64], [33, 31]),
    (1, 1, 128, 256, 16, [16, 500], None),
]


def packed(n, T, H, Hkv, D, dtype, seed):
    x = randn(n, T, H + 2 * Hkv, D, dtype=dtype, g=gen(seed))
    return x[:, :, :H], x[:, :, H:H + Hkv], x[:, :, H + Hkv:]


@pytest.mark.parametrize("style", ["half", "interleaved", None])
@pytest.mark.parametrize("bits", [16, 4])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("shape", APPENDS, ids=lambda s: "x".join(map(str, s[:5])))
def test_append_bit_for_bit(shape, dtype, bits, style):
    """Every row as the formula gives it in fp32, every other byte of the pool and of q_out as it was."""
    H, Hkv, D, ps, T, lens, new = shape
    n, seed = len(lens), 11 * H + D + T
    pool = sum(-(-x // ps) for x in lens) + 2
    table = pg.table_of(lens, ps, pool, np.random.default_rng(seed))
    c = PagedKV(H, Hkv, D, ps, pool, dtype, bits)
    for pages in (c.k_pages, c.v_pages):
        pages.view(torch.uint8).fill_(0x5A)
    want = [p.clone() for p in (c.k_pages, c.v_pages)]
    q, k, v = packed(n, T, H, Hkv, D, dtype, seed)
    news = [min(T, x) for x in lens] if new is None else new
    for b in range(n):                                         # what is padding may hold anything
        k[b, news[b]:], v[b, news[b]:], q[b, news[b]:] = math.nan, math.inf, math.nan
    dev = dict(dtype=torch.int32, device="cuda")
    lens_t, new_t = torch.tensor(lens, **dev), torch.tensor(news, **dev)
    q_out = torch.full((n, T, H, D), 7.0, dtype=dtype, device="cuda")
    want_q = q_out.clone()
    cos = sin = None
    if style:
        cos, sin = (x.cuda() for x in wl.rope_tables(max(lens), D))
    for b in range(n):
        pos = torch.arange(lens[b] - news[b], lens[b], device="cuda")
        kb, vb = k[b, :news[b]], v[b, :news[b]]
        if style:
            kb = pg.turn(kb, cos[pos], sin[pos], style).to(dtype)
            want_q[b, :news[b]] = pg.turn(q[b, :news[b]], cos[pos], sin[pos], style).to(dtype)
        page, off = table[b].cuda()[pos // ps].long(), pos % ps
        for x, pages in ((kb, want[0]), (vb, want[1])):
            if bits == 16:
                pages[page, :, off] = x
            else:
                codes, scales = pg.split4(pages, ps, D, dtype)
                cd, s, z = pg.codes_of(x, dtype)
                codes[page, :, off] = cd[..., 0::2] | (cd[..., 1::2] << 4)
                scales[page, :, off] = torch.cat([s, z], -1)
    new_arg = new_t if new is not None or any(a != T for a in news) else None
    if style:
        got = c.append(k, v, table.cuda(), lens_t, new_arg, q=q, q_out=q_out, rope_cos=cos, rope_sin=sin, style=style)
        assert got is q_out and torch.equal(q_out, want_q)
    else:
        assert c.append(k, v, table.cuda(), lens_t, new_arg) is None
    for got, ref in ((c.k_pages, want[0]), (c.v_pages, want[1])):
        assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8))
    # and back
    rk, rv = (torch.full((n, T, Hkv, D), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    c.read(table.cuda(), lens_t, T, new_arg, rk, rv)
    for b in range(n):
        pos = torch.arange(lens[b] - news[b], lens[b], device="cuda")
        page, off = table[b].cuda()[pos // ps].long(), pos % ps
        for got, pages in ((rk, want[0]), (rv, want[1])):
            if bits == 16:
                ref = pages[page, :, off]
            else:
                codes, scales = pg.split4(pages, ps, D, dtype)
                ref = pg.values4(codes[page, :, off], scales[page, :, off]).to(dtype)
            assert torch.equal(got[b, :news[b]], ref) and (got[b, news[b]:] == 3.0).all()
    assert c.get_error() == 0
    c.destroy()


@pytest.mark.parametrize("style", ["half", "interleaved"])
@pytest.mark.parametrize("D", [64, 256])
def test_rotation_tables_of_any_alignment(D, style):
    table, lens = torch.tensor([[1, 0], [2, -1]], dtype=torch.int32, device="cuda"), torch.tensor([20, 9], dtype=torch.int32, device="cuda")
    q, k, v = packed(2, 9, 4, 2, D, F16, 81)
    tables = [x.cuda() for x in wl.rope_tables(20, D)]
    shifted = []
    for x in tables:
        flat = torch.empty(x.numel() + 1, device="cuda")[1:]
        shifted.append(flat.view_as(x).copy_(x))
    got = []
    for cos, sin in (tables, shifted, (tables[0], shifted[1])):
        c = PagedKV(4, 2, D, 16, 3, F16, 16)
        c.k_pages.zero_()
        got.append((c.append(k, v, table, lens, q=q, rope_cos=cos, rope_sin=sin, style=style), c.k_pages.clone()))
        c.destroy()
    for q_out, pages in got[1:]:
        assert torch.equal(q_out, got[0][0]) and torch.equal(pages, got[0][1])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [2.0 ** -20, 1.0, 2.0 ** 9])
def test_codes_of_values_halfway_between_two(dtype, scale):
    """Values on, and one unit beside, the middle between two codes: the rounded quotient decides, ties to even."""
    n, D, ps = 64, 128, 64
    rng = np.random.default_rng(17)
    c = PagedKV(4, 4, D, ps, n, dtype, 4)
    step = torch.from_numpy(rng.integers(128, 256, (n * ps, 1, 1, 4)) * scale / 64.0)
    k = torch.from_numpy(rng.integers(-8, 8, (n * ps, 4, D // 4, 4)) + 0.5 * rng.integers(0, 2, (n * ps, 4, D // 4, 4)))
    k[:, :, 0], k[:, :, 1] = -8, 7                             # (the whole range, so that the scale is the step or its neighbour)
    x = (step * k + torch.from_numpy(rng.integers(-40, 40, (n * ps, 4, 1, 4))) * step / 8).to(dtype).flatten(-2)
    side = torch.from_numpy(rng.integers(-1, 2, x.shape)).to(torch.int16)
    x = (x.view(torch.int16) + torch.where(x == 0, torch.zeros_like(side), side)).view(dtype).cuda().view(n, ps, 4, D)
    table = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1)
    c.append(x, x, table, torch.full((n,), ps, dtype=torch.int32, device="cuda"))
    codes, scales = pg.split4(c.k_pages, ps, D, dtype)
    cd, s, z = pg.codes_of(x.transpose(1, 2), dtype)
    assert torch.equal(scales, torch.cat([s, z], -1)) and torch.equal(codes, cd[..., 0::2] | (cd[..., 1::2] << 4))
    assert torch.equal(c.k_pages, c.v_pages) and c.get_error() == 0
    c.destroy()


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_four_bit_rows_at_the_edges(dtype):
    """Constant rows, zeros, the smallest and largest values, Inf and NaN in one group of four."""
    D, ps = 128, 16
    c = PagedKV(1, 1, D, ps, 1, dtype, 4)
    top = torch.finfo(dtype).max
    k = randn(1, 16, 1, D, dtype=dtype, g=gen(81))
    k[0, 0] = 0
    k[0, 1] = 1.5
    k[0, 2] = -0.0
    k[0, 3, 0, 5], k[0, 4, 0, 6], k[0, 5, 0, 127] = math.nan, math.inf, -math.inf
    k[0, 6] *= 2.0 ** -12
    k[0, 7, 0, ::2], k[0, 7, 0, 1::2] = 60000.0, -60000.0
    k[0, 8, 0, 0], k[0, 8, 0, 4] = top, -top                   # fp16: held; bf16: a range that fp32 has no room for
    k[0, 9] += 1000
    table, lens = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.full((1,), 16, dtype=torch.int32, device="cuda")
    c.append(k, k, table, lens)
    codes, scales = pg.split4(c.k_pages, ps, D, dtype)
    cd, s, z = pg.codes_of(k[0].transpose(0, 1), dtype)
    assert torch.equal(codes[0], cd[..., 0::2] | (cd[..., 1::2] << 4))
    ref = torch.cat([s, z], -1)
    assert torch.equal(torch.isnan(scales[0]), torch.isnan(ref)) and torch.equal(scales[0].nan_to_num(0.0), ref.nan_to_num(0.0))
    rk, _ = c.read(table, lens, 16)
    assert torch.equal(rk[0, 1], k[0, 1]) and not rk[0, 0].any()
    g = torch.isnan(rk[0, 3, 0]).unflatten(0, (-1, 4))
    assert g[:, 1].all() and not g[:, [0, 2, 3]].any()
    # half a step, and what rounding the scale (15 steps of it) and the zero point leaves
    u = torch.finfo(dtype).eps / 2
    for i in (6, 9, 10, 11, 12, 13, 14, 15):
        step = s[0, i].double().repeat(D // 4)
        off = z[0, i].double().abs().repeat(D // 4)
        bound = step * (0.5 + 16 * u) + off * 2 * u + k[0, i, 0].double().abs() * u + 2.0 ** -24
        assert ((rk[0, i, 0].double() - k[0, i, 0].double()).abs() <= bound).all()
    c.destroy()


def test_queries_rotated_in_place():
    c = PagedKV(4, 2, 64, 16, 4, F16)
    q, k, v = (randn(2, 5, h, 64, dtype=F16, g=gen(91 + h)) for h in (4, 2, 2))
    table, lens = torch.tensor([[0], [1]], dtype=torch.int32, device="cuda"), torch.tensor([9, 5], dtype=torch.int32, device="cuda")
    cos, sin = (x.cuda() for x in wl.rope_tables(9, 64))
    want = c.append(k, v, table, lens, q=q, rope_cos=cos, rope_sin=sin)
    assert c.append(k, v, table, lens, q=q, q_out=q, rope_cos=cos, rope_sin=sin) is q
    assert torch.equal(q, want)
    c.destroy()


# ---------------------------------------------------------------------------------------- what only the device can see
@pytest.mark.parametrize("bits", [16, 4])
def test_bad_tables_are_flagged(bits):
    c, table, lens = filled(4, 2, 64, 16, [30, 40], F16, bits, 101)
    before = [p.clone() for p in (c.k_pages, c.v_pages)]
    q = randn(2, 1, 4, 64, dtype=F16, g=gen(102))
    good = c.sdpa(q, table, lens)
    for value in (-1, c.num_pages, 2 ** 31 - 1, -2 ** 31):
        bad = table.clone()
        bad[1, 1] = value
        out = c.sdpa(q, bad, lens)
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE and torch.equal(out[0], good[0]) and torch.isfinite(out[1]).all()
        c.read(bad, lens, 40)
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE
        k = randn(2, 3, 2, 64, dtype=F16, g=gen(103))
        at = torch.tensor([3, 19], dtype=torch.int32, device="cuda")
        c.append(k, k, bad, at, torch.tensor([0, 3], dtype=torch.int32, device="cuda"))         # positions 16-18 have no page
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE
        assert all(torch.equal(a, b) for a, b in zip(before, (c.k_pages, c.v_pages)))
    for value in (-5, 49, 2 ** 31 - 1, -2 ** 31):
        out = c.sdpa(q, table, torch.tensor([30, value], dtype=torch.int32, device="cuda"))
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE and torch.equal(out[0], good[0])
        assert not out[1].any() if value < 0 else torch.isfinite(out[1]).all()
        c.append(k, k, table, torch.tensor([0, value], dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE
        assert all(torch.equal(a, b) for a, b in zip(before, (c.k_pages, c.v_pages)))
    c.destroy()


@pytest.mark.parametrize("bits", [16, 4])
def test_bad_tables_are_flagged_where_rows_are_many(bits):
    c, table, lens = filled(4, 2, 64, 16, [300, 280], F16, bits, 105)
    q = randn(2, 256, 4, 64, dtype=F16, g=gen(106))
    good = c.sdpa(q, table, lens)
    for value in (-1, c.num_pages, 2 ** 31 - 1, -2 ** 31):
        bad = table.clone()
        bad[1, 3] = value
        out = c.sdpa(q, bad, lens)
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE and torch.equal(out[0], good[0]) and torch.isfinite(out[1]).all()
    for value in (-5, 305, 2 ** 31 - 1, -2 ** 31):
        out = c.sdpa(q, table, torch.tensor([300, value], dtype=torch.int32, device="cuda"))
        assert c.get_error() == sk.SEGKV_DEV_BAD_PAGE and torch.equal(out[0], good[0])
        assert not out[1].any() if value < 0 else torch.isfinite(out[1]).all()
    c.destroy()


def test_positions_behind_the_rotation_tables_are_flagged():
    c = PagedKV(2, 1, 64, 16, 2, F16)
    cos, sin = (x.cuda() for x in wl.rope_tables(8, 64))
    q, k = randn(1, 4, 2, 64, dtype=F16, g=gen(111)), randn(1, 4, 1, 64, dtype=F16, g=gen(112))
    table, lens = torch.tensor([[1]], dtype=torch.int32, device="cuda"), torch.tensor([10], dtype=torch.int32, device="cuda")
    q_out = torch.full_like(q, 5.0)
    c.append(k, k, table, lens, q=q, q_out=q_out, rope_cos=cos, rope_sin=sin)          # positions 6 to 9 of 8
    assert c.get_error() == sk.SEGKV_DEV_BAD_POSITION and c.get_error() == 0
    assert (q_out[0, 2:] == 5.0).all() and (q_out[0, :2] != 5.0).any()
    assert c.k_pages[1, 0, 6:8].any(-1).all() and not c.k_pages[1, 0, 8:].any()
    c.destroy()


# ----------------------------------------------------------------------------------------------------- as it is used
@pytest.mark.parametrize("bits", [16, 4])
def test_captured_step_follows_the_lengths(bits):
    """One captured append and attention, replayed while the lengths grow, against the same calls made one by one."""
    H, Hkv, D, ps, n = 8, 2, 128, 16, 3
    start = [15, 100, 0]
    pool = 40
    rng = np.random.default_rng(5)
    table = torch.from_numpy(rng.permutation(pool)[:n * 8].reshape(n, 8).astype(np.int32)).cuda()
    cos, sin = (x.cuda() for x in wl.rope_tables(128, D))
    caches = [PagedKV(H, Hkv, D, ps, pool, BF16, bits) for _ in range(2)]
    k0, v0 = (randn(n, 100, Hkv, D, dtype=BF16, g=gen(121 + i)) for i in range(2))
    lens = torch.tensor(start, dtype=torch.int32, device="cuda")
    for c in caches:
        c.append(k0, v0, table, lens, lens)
    q, k, v = (torch.zeros(n, 1, h, D, dtype=BF16, device="cuda") for h in (H, Hkv, Hkv))
    qr, out = torch.zeros_like(q), torch.zeros_like(q)

    def step(c, qr, out):
        c.append(k, v, table, lens, q=q, q_out=qr, rope_cos=cos, rope_sin=sin)
        c.sdpa(qr, table, lens, out)

    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(caches[0], qr, out)
    for t in range(20):
        for i, x in enumerate((q, k, v)):
            x.copy_(randn(*x.shape, dtype=BF16, g=gen(130 + 3 * t + i)))
        lens += 1
        if t == 7:
            lens[1] = 0                                        # a request has left
        g.replay()
        qr2, out2 = torch.zeros_like(q), torch.zeros_like(q)
        step(caches[1], qr2, out2)
        torch.cuda.synchronize()
        live = lens > 0
        assert torch.equal(qr[live], qr2[live]) and torch.equal(out, out2)
        if t in (0, 6, 7, 19):
            pg.check(out, *pg.attention(caches[1], qr2, table, lens.tolist()))
    assert [c.get_error() for c in caches] == [0, 0]
    for c in caches:
        c.destroy()


def test_from_prompt_to_pages_to_beams():
    """A prompt attended to by the segment cache's prefill and stored in pages, steps served from them, the sequence read back into a
    segment cache and continued there: the same attention from either."""
    H, Hkv, D, ps, P = 8, 2, 128, 32, 75
    w = wl.Workload("handover", 2, 1, H, Hkv, D, P, 4, "f16", "uniform", False, 300)
    k, v = wl.make_prompt(w, "cuda")
    lens = [P, 41]
    h = sk.SegKV(2, 1, H, Hkv, D, P + 8, 8, F16)
    h.prefill_write_ragged(k, v, lens)
    qp = wl.make_prefill_query(w, "cuda")
    out_p = h.prefill_sdpa(qp, torch.zeros_like(qp))
    c = PagedKV(H, Hkv, D, ps, 12, F16)
    table = pg.table_of([P + 8, 49], ps, 12, np.random.default_rng(3)).cuda()
    n_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.append(k, v, table, n_lens, n_lens)
    # the prompt's own attention over the pages is the prefill's
    for b in range(2):
        one = c.sdpa(qp[b:b + 1, :lens[b]].contiguous(), table[b:b + 1].contiguous(), n_lens[b:b + 1].contiguous())
        ref, tol = pg.attention(c, qp[b:b + 1, :lens[b]], table[b:b + 1], lens[b:b + 1])
        pg.check(one, ref, tol)
        pg.check(out_p[b:b + 1, :lens[b]], ref, 2e-3 + 1e-2 * ref.abs())
    for t in range(3):
        q, kn, vn = wl.make_step(w, t, "cuda")
        n_lens += 1
        c.append(kn.unsqueeze(1), vn.unsqueeze(1), table, n_lens)
        a = c.sdpa(q.unsqueeze(1), table, n_lens)
        b = h.decode_step(t, torch.zeros(2, dtype=torch.int32, device="cuda") if t else None, kn, vn, q)
        ref, tol = pg.attention(c, q.unsqueeze(1), table, n_lens.tolist())
        pg.check(a, ref, tol)
        pg.check(b.unsqueeze(1), ref, 2e-3 + 1e-2 * ref.abs())
    longest = int(n_lens.max())
    rk, rv = c.read(table, n_lens, longest, n_lens)
    beams = sk.SegKV(2, 4, H, Hkv, D, longest, 4, F16)
    beams.prefill_write_ragged(rk, rv, n_lens.tolist())
    q = randn(8, H, D, dtype=F16, g=gen(140))
    got = beams.decode_sdpa(q)
    for j in range(4):
        rows = torch.stack([q[j], q[4 + j]]).unsqueeze(1)
        ref, _ = pg.attention(c, rows, table, n_lens.tolist())
        pg.check(torch.stack([got[j], got[4 + j]]).unsqueeze(1), ref, 2e-3 + 1e-2 * ref.abs())
    for x in (h, c, beams):
        x.destroy()


@pytest.mark.parametrize("bits", [16, 4])
def test_other_streams_and_layers_in_a_row(bits):
    """Two layers' calls one behind the other on a side stream, with and without overlap, give what calls that are waited for give."""
    H, Hkv, D, ps = 4, 2, 64, 16
    lens = [200, 31]
    sets = [filled(H, Hkv, D, ps, lens, F16, bits, 150 + i) for i in range(2)]
    cos, sin = (x.cuda() for x in wl.rope_tables(200, D))
    q, k, v = (randn(2, 1, h, D, dtype=F16, g=gen(160 + h)) for h in (H, Hkv, Hkv))

    def chain(stream, wait):
        x, outs = q, []
        for c, table, n_lens in sets * 3:
            x = c.append(k, v, table, n_lens, q=x, rope_cos=cos, rope_sin=sin, stream=stream)
            if wait:
                torch.cuda.synchronize()
            x = c.sdpa(x, table, n_lens, stream=stream)
            if wait:
                torch.cuda.synchronize()
            outs.append(x)
        torch.cuda.synchronize()
        return outs

    want = chain(None, True)
    st = torch.cuda.Stream()
    for overlap in (True, False):
        for c, _, _ in sets:
            c.set_overlap(overlap)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            got = chain(None if overlap else st, False)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    for c, _, _ in sets:
        c.destroy()


def test_refused_arguments():
    c, table, lens = filled(4, 2, 64, 16, [30, 40], F16, 16, 171)
    q = randn(2, 1, 4, 64, dtype=F16, g=gen(172))
    k = randn(2, 1, 2, 64, dtype=F16, g=gen(173))
    cos, sin = (x.cuda() for x in wl.rope_tables(64, 64))
    n0 = c.launch_count
    for bad in (q.float(), q.cpu(), q[:1], q[..., :32], q[:, :, :2], q[:, 0], q.transpose(1, 2),
                torch.zeros(2, 1, 4, 65, dtype=F16, device="cuda")[..., :64]):
        with pytest.raises(ValueError):
            c.sdpa(bad, table, lens)
    for bad in (table.long(), table.cpu(), table[:1], table[:, 0], table.t()):
        with pytest.raises(ValueError):
            c.sdpa(q, bad, lens)
    for bad in (lens.long(), lens.cpu(), lens[:1], lens[:, None]):
        with pytest.raises(ValueError):
            c.sdpa(q, table, bad)
    with pytest.raises(ValueError):
        c.sdpa(q, table, lens, torch.zeros_like(q).float())
    with pytest.raises(ValueError):
        c.sdpa(q, table, lens, None, torch.ones(3, device="cuda"))
    for kw in (dict(q=q), dict(q=q, rope_cos=cos), dict(q_out=q), dict(rope_cos=cos, rope_sin=sin[:3]), dict(rope_cos=cos.half(), rope_sin=sin.half()),
               dict(rope_cos=cos, rope_sin=sin, style=7)):
        with pytest.raises((ValueError, sk.SegKVError)):
            c.append(k, k, table, lens, **kw)
    with pytest.raises(ValueError):
        c.append(k, k[:, :0], table, lens)
    with pytest.raises(ValueError):
        c.append(torch.zeros(2, 1, 2, 64, dtype=F16, device="cuda").expand(2, 1, 2, 64)[:, :, :1], k, table, lens)
    with pytest.raises(ValueError):
        c.read(table, lens, 3, k=torch.zeros(2, 2, 2, 64, dtype=F16, device="cuda"))
    with pytest.raises(ValueError):                            # rows that start off a 16-byte boundary
        c.append(torch.zeros(2, 1, 2 * 64 + 4, dtype=F16, device="cuda")[..., :128].unflatten(-1, (2, 64)), k, table, lens)
    with pytest.raises(sk.SegKVError):
        c.append(torch.zeros(2 * 2 * 64 + 4, dtype=F16, device="cuda")[4:].view(2, 1, 2, 64), k, table, lens)
    assert c.launch_count == n0
    # nothing to do is done
    c.sdpa(q[:, :0], table, lens)
    c.append(k[:, :0], k[:, :0], table, lens)
    c.read(table, lens, 0)
    assert c.launch_count == n0 and c.get_error() == 0
    for kw in (dict(k_pages=c.k_pages), dict(k_pages=c.k_pages.float(), v_pages=c.v_pages.float()), dict(k_pages=c.k_pages[:2], v_pages=c.v_pages[:2])):
        with pytest.raises(ValueError):
            PagedKV(4, 2, 64, 16, c.num_pages, F16, 16, **kw)
    c.destroy()
    with pytest.raises(sk.SegKVError):
        c.sdpa(q, table, lens)


def test_calls_with_a_stream_argument_take_the_general_path():
    """The same calls through the extension module and through ctypes: what one takes the other takes, with the same bits."""
    c, table, lens = filled(4, 2, 64, 16, [30, 40], F16, 4, 181)
    st = torch.cuda.current_stream()
    q, k, v = packed(2, 2, 4, 2, 64, F16, 182)
    cos, sin = (x.cuda() for x in wl.rope_tables(64, 64))
    new = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    got = []
    for stream in (None, st):
        qr = c.append(k, v, table, lens, new, q=q, q_out=torch.zeros(2, 2, 4, 64, dtype=F16, device="cuda"), rope_cos=cos, rope_sin=sin,
                      style="interleaved", stream=stream)
        got.append([qr, c.sdpa(qr, table, lens, None, wl.alibi_slopes(4).cuda(), stream=stream), *c.read(table, lens, 3, new, stream=stream)])
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert c._hot is None or c._hot.sdpa(q.float(), table, lens, got[0][1], None) is None       # not its to take
    c.destroy()
