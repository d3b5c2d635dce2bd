"""Few rows times FB4 weights and the 8-bit cache, against plain forms in float64 (and integers)."""

import math
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

INF = math.inf
BF16 = 2.0 ** -8     # half a step of bf16, relative
FP32 = 2.0 ** -24


@pytest.fixture(scope="module")
def F():
    import paper_2603_02883_amd as F
    assert torch.cuda.is_available()
    return F


@pytest.fixture(scope="module")
def luts(F, fbk):
    return F.fb4_build_luts(fbk)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ few rows times weights
def weights(F, luts, g, n, cols, block, size=1.0):
    w = randn(g, n, cols) * torch.exp(randn(g, n, 1)) * size
    return F.fb4_quantize(luts, F.opts(block=block), w.bfloat16())


def check_product(F, luts, x, codes, meta, block, bias, out):
    w = F.fb4_dequantize(luts, codes, meta, block=block, out_dtype=F.DTYPE_F32).double()
    y, size = x.double() @ w.T, x.double().abs() @ w.abs().T
    if bias is not None:
        y, size = y + bias.double(), size + bias.double().abs()
    # products of two bf16 are exact in fp32; every addition rounds once, to a sum that the sizes' bounds
    tol = (x.shape[1] + 10) * FP32 * size + (BF16 * y.abs() if out.dtype is torch.bfloat16 else 0.0)
    fine = torch.isfinite(y)
    assert torch.equal(torch.isfinite(out), fine), "not finite elsewhere"
    err = (out.double() - y).abs()
    worst = (err - tol)[fine].max().item() if fine.any() else 0.0
    assert worst <= 0, (worst, err[fine].max().item())


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("rows,n,cols", [(1, 1, 32), (1, 17, 64), (2, 16, 96), (15, 130, 288), (16, 1152, 1152), (17, 100, 4608), (31, 33, 256), (33, 4611, 1184),
                                         (64, 1000, 512), (49, 15, 32), (1, 8200, 1152), (5, 32800, 96), (16, 33000, 64), (20, 33000, 64), (64, 33000, 160), (3, 8200, 16384)])
def test_products(F, luts, rows, n, cols, block):
    g = gen(rows * 7 + n)
    codes, meta = weights(F, luts, g, n, cols, block)
    x, bias = randn(g, rows, cols).bfloat16(), randn(g, n)
    for b, dtype in ((bias, F.DTYPE_F32), (None, F.DTYPE_BF16), (bias, F.DTYPE_BF16)):
        out = F.fb4_matvec(luts, x, codes, meta, block=block, bias=b, out_dtype=dtype)
        assert out.dtype is (torch.float32 if dtype == F.DTYPE_F32 else torch.bfloat16)
        check_product(F, luts, x, codes, meta, block, b, out)


@pytest.mark.parametrize("size", [2.0 ** -118, 2.0 ** -60, 2.0 ** 110])
def test_products_with_scales_at_the_ends(F, luts, size):
    g = gen(3)
    codes, meta = weights(F, luts, g, 40, 96, 32, size)
    x = (randn(g, 7, 96) * min(1.0, 2.0 ** 10 / size) * (2.0 ** 60 if size < 2.0 ** -100 else 1.0)).bfloat16()
    check_product(F, luts, x, codes, meta, 32, None, F.fb4_matvec(luts, x, codes, meta, out_dtype=F.DTYPE_F32))


def test_products_views_and_rows_that_are_no_numbers(F, luts):
    g = gen(4)
    codes, meta = weights(F, luts, g, 77, 320, 32)
    wide = randn(g, 20, 640).bfloat16()
    x = wide[:, 320:]
    x[3, 5], x[7, 0], x[19, 319] = math.nan, INF, -INF
    held = torch.full((20, 100), 7.0, device="cuda")
    out = held[:, 10:87]
    F.fb4_matvec(luts, x, codes, meta, out=out)
    live = [i for i in range(20) if i not in (3, 7, 19)]
    check_product(F, luts, x[live], codes, meta, 32, None, out[live])
    assert out[3].isnan().all()
    w = F.fb4_dequantize(luts, codes, meta).double()
    for row, c, sign in ((7, 0, 1), (19, 319, -1)):   # Inf times a weight, NaN where that is 0
        want = torch.where(w[:, c] == 0, math.nan, sign * INF * w[:, c])
        assert torch.equal(out[row].double().nan_to_num(nan=5.0), want.nan_to_num(nan=5.0)), row
    assert (held[:, :10] == 7).all() and (held[:, 87:] == 7).all()


def test_products_of_dialects_that_are_none_and_empty_ones(F, fbk):
    few = F.fb4_build_luts(fbk[:3])
    g = gen(5)
    codes = torch.randint(0, 256, (30, 64), device="cuda", generator=g, dtype=torch.uint8)
    meta = torch.randint(0, 256, (30, 4), device="cuda", generator=g, dtype=torch.int16) + 127 * 256
    x = randn(g, 4, 128).bfloat16()
    out = F.fb4_matvec(few, x, codes, meta, out_dtype=F.DTYPE_F32)
    check_product(F, few, x, codes, meta, 32, None, out)
    bias = randn(g, 30)
    none = F.fb4_matvec(few, x[:, :0], codes[:, :0], meta[:, :0], bias=bias, out_dtype=F.DTYPE_F32)
    assert torch.equal(none, bias.expand(4, 30))
    assert F.fb4_matvec(few, x[:0], codes, meta).shape == (0, 30) and F.fb4_matvec(few, x, codes[:0], meta[:0]).shape == (4, 0)


# ------------------------------------------------------------------------------------------------ plan
def plan_plain(lens, adds, tables, free, count, page, tokens):
    """Sequence by sequence, on Python lists."""
    wide, n_free = len(tables[0]) if tables else 0, len(free)
    pages = lambda n: -(-n // page)
    lens = [min(max(n, 0), wide * page) for n in lens]
    count = min(max(count, 0), n_free)
    stack = free[:count]
    free, tables = list(free), [list(t) for t in tables]
    at = count
    for b, a in enumerate(adds):
        if a < 0:
            new = max(lens[b] + a, 0)
            for p in range(pages(new), pages(lens[b])):
                if at < n_free:
                    free[at] = tables[b][p]
                    stack.append(tables[b][p])
                at += 1
            lens[b] = new
    starts, slots, positions, open_ = [0], [], [], True
    for b, a in enumerate(adds):
        if a > 0 and lens[b] + a <= wide * page and open_:
            need = pages(lens[b] + a) - pages(lens[b])
            if need > len(stack) or starts[-1] + a > tokens:
                open_ = False
            else:
                for p in range(pages(lens[b]), pages(lens[b] + a)):
                    tables[b][p] = stack.pop()
                for i in range(lens[b], lens[b] + a):
                    p = tables[b][i // page]
                    slots.append(p * page + i % page if 0 <= p and (p + 1) * page <= 2 ** 31 else -1)
                    positions.append(i)
                lens[b] += a
        starts.append(len(slots))
    slots += [-1] * (tokens - len(slots))
    positions += [0] * (tokens - len(positions))
    return dict(lens=lens, count=[len(stack)], starts=starts, slots=slots, positions=positions, tables=tables, free=free)


def check_plan(F, lens, adds, tables, free, count, page, tokens, in_place=False, positions=True):
    t = dict(lens=ints(lens), adds=ints(adds), tables=ints(tables).view(len(lens), len(tables[0]) if tables else 0), free=ints(free), count=ints([count]))
    more = dict(lens_out=t["lens"], free_count_out=t["count"]) if in_place else {}
    got = F.fb4_cache_plan(t["lens"], t["adds"], t["tables"], t["free"], t["count"], page, tokens, **more)
    want = plan_plain(lens, adds, tables, free, count, page, tokens)
    got = dict(zip(("lens", "count", "starts", "slots", "positions"), got), tables=t["tables"], free=t["free"])
    for name, x in got.items():
        assert x.cpu().tolist() == want[name], name
    if not in_place:
        again = F.fb4_cache_plan(t["lens"], t["adds"], t["tables"], t["free"], t["count"], page, tokens)
        assert all(torch.equal(a, got[n]) for a, n in zip(again, ("lens", "count", "starts", "slots", "positions")))
    return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,page,room", [(1, 16, 1.0), (3, 32, 1.0), (64, 64, 1.0), (65, 16, 0.6), (300, 128, 0.5), (1000, 16, 1.0), (4096, 16, 0.7), (17, 64, 0.0)])
def test_plans(F, batch, page, room, in_place):
    r = random.Random(batch + page)
    wide = 9
    lens = [r.randint(0, wide * page) for _ in range(batch)]
    adds = [r.choice([1, 1, 0, r.randint(1, 3 * page), -r.randint(1, 2 * page), -10 ** 6]) for _ in range(batch)]
    ids = list(range(10 ** 6, 10 ** 6 + batch * wide))
    r.shuffle(ids)
    tables = [[ids.pop() if p * page < lens[b] else -1 for p in range(wide)] for b in range(batch)]
    count = int(len(ids) * room)
    free = ids[:count] + [-5] * (batch * wide - count)
    tokens = sum(max(a, 0) for a in adds)
    want = check_plan(F, lens, adds, tables, free, count, page, tokens + 7, in_place)
    assert want["starts"][-1] > 0 or room == 0 or batch == 1
    check_plan(F, lens, adds, tables, free, count, page, tokens // 2, in_place)     # (rows run out)
    check_plan(F, lens, adds, tables, free[:count + 1], count, page, tokens, in_place)   # (what comes back finds no room)


def test_plans_at_the_ends(F):
    check_plan(F, [], [], [], [3, 4], 2, 16, 0)
    check_plan(F, [], [], [], [], 0, 16, 5)
    check_plan(F, [-5, 10 ** 9, 0], [3, 1, 2], [[-1, -1], [7, 8], [-1, -1]], [1, 2, 3], 99, 16, 10)      # lengths and counts that are none
    check_plan(F, [0, 0], [33, 4], [[-1, -1], [-1, -1]], [1, 2, 3], 3, 16, 100)                            # one that would pass its table by itself
    check_plan(F, [0, 0], [2 ** 31 - 1, 4], [[-1, -1], [-1, -1]], [1, 2, 3], 3, 16, 100)
    check_plan(F, [5, 5], [-2 ** 31, 1], [[4, -1], [5, -1]], [1, 2, 3], 1, 16, 100)
    check_plan(F, [16, 16], [1, 1], [[4, -1], [5, -1]], [-1, 2 ** 27], 2, 16, 4)                           # pages without slots
    check_plan(F, [16, 16], [1, 1], [[4, -1], [5, -1]], [-1, 2 ** 27 - 1], 2, 16, 4)


def test_plans_of_many_tokens(F):
    r = random.Random(9)
    page, batch, wide = 64, 20, 80
    lens = [r.randint(0, 1000) for _ in range(batch)]
    adds = [r.randint(0, 4000) for _ in range(batch)]
    ids = list(range(batch * wide))
    tables = [[ids.pop() if p * page < lens[b] else -1 for p in range(wide)] for b in range(batch)]
    for tokens in (16384, 16385, sum(adds), sum(adds) + 1000):
        check_plan(F, lens, adds, tables, ids, len(ids), page, tokens)
        check_plan(F, lens, adds, tables, ids, len(ids), page, tokens, in_place=True)


# ------------------------------------------------------------------------------------------------ store
def e4m3(x):
    """Four significant bits, exponents from 2^-6 on, multiples of 2^-9 below; ties to even; NaN for what is no number.  Of float64."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    y = np.where(fine, x, 0.0)
    _, e = np.frexp(y)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.where(fine, np.round(y / step) * step, np.nan)


def values_of(cache):
    """float64 numpy of E4M3 bytes, read bit by bit."""
    b = cache.cpu().numpy().astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.ldexp(1.0, e - 10))
    return np.where(b >> 7 == 1, -1.0, 1.0) * np.where(b & 0x7F == 0x7F, np.nan, v)


def store_plain(k, v, slots, cache, scales, page):
    """Page by page: the values and scale bytes that a store leaves."""
    _, pages, heads, size = cache.shape
    dim = size // page
    held, scales = values_of(cache), scales.cpu().numpy().astype(np.int64)
    x = [t.double().cpu().numpy() for t in (k, v)]
    by_page = {}
    for t, s in enumerate(slots):
        if 0 <= s < pages * page:
            by_page.setdefault(s // page, {})[s % page] = t     # (the last one stays)
    for p, place in by_page.items():
        at, tokens = list(place), list(place.values())
        for which in range(2):
            for h in range(heads):
                rows = x[which][h][tokens]
                top = np.abs(np.where(np.isfinite(rows), rows, 0.0)).max()
                e = -117
                while top > 448 * 2.0 ** e:
                    e += 1
                to = held[which, p, h].reshape(page, dim) if which == 0 else held[which, p, h].reshape(dim, page).T
                if 0 not in place:
                    old = scales[which, p, h] - 127
                    if e > old:
                        to[:] = e4m3(to * 2.0 ** (old - e))
                    e = max(e, old)
                to[at] = e4m3(rows / 2.0 ** e)
                scales[which, p, h] = e + 127
    return held, scales


def new_cache(g, pages, heads, dim, page):
    """Pages with something in them: any finite elements, scales of a usual size."""
    cache = torch.randint(0, 256, (2, pages, heads, page * dim), device="cuda", generator=g, dtype=torch.uint8)
    cache[(cache & 0x7F) == 0x7F] = 1
    scales = torch.randint(110, 125, (2, pages, heads), device="cuda", generator=g, dtype=torch.int32).to(torch.uint8)
    return cache, scales


def check_store(F, k, v, slots, cache, scales, page):
    want, want_scales = store_plain(k, v, slots, cache, scales, page)
    F.fb4_cache_store(k, v, ints(slots), cache, scales, page)
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    got = values_of(cache)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    assert same.all(), np.argwhere(~same)[:5]


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [8, 24, 64, 72, 128])
def test_stores(F, page, dim):
    g, heads, pages = gen(page + dim), 3, 40
    cache, scales = new_cache(g, pages, heads, dim, page)
    k, v = (randn(g, heads, 5 * page + 9, dim) * torch.exp(2 * randn(g, heads, 5 * page + 9, 1)) for _ in range(2))
    k, v = k.bfloat16(), v.bfloat16()
    at = list(range(7 * page, 9 * page + 5))                     # whole pages and a begun one
    at += list(range(3 * page + 7, 4 * page))                    # the end of a begun one
    at += [20 * page + 3, 21 * page, -1, 22 * page + page - 1]   # single tokens, one without a place
    at += list(range(25 * page + 1, 25 * page + 12))
    at += [pages * page, 2 ** 31 - 1, -2 ** 31, 30 * page + 2]   # slots that are none
    for many in (len(at), 1):
        check_store(F, k[:, :many], v[:, :many], at[:many], cache, scales, page)
    # token by token onto the same page
    for i in range(6):
        check_store(F, k[:, 50 + i:51 + i] * 4 ** i, v[:, 50 + i:51 + i] * 4 ** i, [33 * page + i], cache, scales, page)


@pytest.mark.parametrize("page", [16, 64])
def test_stores_of_many_tokens(F, page):
    """Enough for workgroups of several tokens each, runs that cross their borders."""
    g, heads, dim, pages = gen(1), 2, 40, 200
    cache, scales = new_cache(g, pages, heads, dim, page)
    r = random.Random(page)
    at = []
    for p in r.sample(range(pages), 150):
        a, n = r.choice([(0, page), (r.randrange(page), page), (0, r.randint(1, page))])
        at += range(p * page + a, min(p * page + page, p * page + a + n))
    k, v = randn(g, heads, len(at), dim).bfloat16(), randn(g, heads, len(at), dim).bfloat16()
    check_store(F, k, v, at, cache, scales, page)


def test_stores_of_one_slot_twice(F):
    """The last of several tokens for a slot is the one that stays, and counts for the scale."""
    g, page, dim = gen(2), 16, 32
    cache, scales = new_cache(g, 4, 2, dim, page)
    at = [16 + 3, 16 + 3, 16 + 4, 16 + 3, 32, 32, 33] + [48 + 1] * 600
    k, v = randn(g, 2, len(at), dim).bfloat16(), randn(g, 2, len(at), dim).bfloat16()
    k[:, 0] *= 1024
    check_store(F, k, v, at, cache, scales, page)


def test_stores_of_values_at_the_ends(F):
    """Zeros, subnormals, the largest numbers, Inf and NaN, magnitudes around 448 times a power of two."""
    g, page, dim, heads = gen(6), 16, 16, 1
    cache, scales = new_cache(g, 12, heads, dim, page)
    rows = torch.zeros(heads, 12, dim)
    rows[0, 1], rows[0, 2, 3], rows[0, 3, 0] = 2.0 ** -133, 3.3895313892515355e38, 2.0 ** -126
    rows[0, 4, :3] = torch.tensor([INF, 1.0, -2.0])
    rows[0, 5, :3] = torch.tensor([math.nan, 448.0, -450.0])
    rows[0, 6], rows[0, 7, 0], rows[0, 8, 0] = INF, 1.75, 1.7578125
    rows[0, 9, :4] = torch.tensor([-448.0, 0.0146484375, 0.0009765625, 0.00146484375])
    rows[0, 10, 0], rows[0, 11, 0] = -0.0, 1.0
    k = rows.bfloat16().cuda()
    for first in (0, 3):   # pages begun anew, and ones that hold something
        check_store(F, k, k.flip(2), [p * page + first for p in range(12)], cache, scales, page)


def test_stores_of_views(F):
    g, page, dim, heads, tokens = gen(8), 32, 64, 4, 70
    packed = randn(g, tokens, 3 * heads, dim).bfloat16()
    k, v = packed[:, heads:2 * heads].transpose(0, 1), packed[:, 2 * heads:].transpose(0, 1)
    for k_, v_ in ((k, v), (k.contiguous(), v), (k[:, :1].expand(-1, tokens, -1), v)):
        cache, scales = new_cache(g, 5, heads, dim, page)
        check_store(F, k_, v_, list(range(40, 40 + tokens)), cache, scales, page)


# ------------------------------------------------------------------------------------------------ attention
class Paged:
    """A cache of sequences with random pages: held values, and what lies behind a sequence's end is NaN."""

    def __init__(self, F, seed, lens, heads_k, dim, page, spare=3, wide=None, scale_spread=6):
        g = gen(seed)
        need = [-(-n // page) for n in lens]
        self.pages, self.page, self.dim, self.heads_k, self.lens_list = sum(need) + spare, page, dim, heads_k, list(lens)
        self.cache, _ = new_cache(g, self.pages, heads_k, dim, page)
        self.scales = (torch.randint(0, scale_spread, (2, self.pages, heads_k), device="cuda", generator=g, dtype=torch.int32) + 118 - scale_spread // 2).to(torch.uint8)
        order = torch.randperm(self.pages, device="cuda", generator=g).tolist()
        self.tables = torch.full((len(lens), max(need + [0]) + 2 if wide is None else wide), -7, dtype=torch.int32, device="cuda")
        for b, n in enumerate(need):
            mine = [order.pop() for _ in range(n)]
            self.tables[b, :n] = ints(mine)
            if lens[b] % page:
                rest = lens[b] % page
                self.cache[0, mine[-1]].view(heads_k, page, dim)[:, rest:] = 0x7F
                self.cache[1, mine[-1]].view(heads_k, dim, page)[:, :, rest:] = 0xFF
        self.lens = ints(self.lens_list)

    def values(self, b):
        """(keys, values) float64 [heads_k][len][dim], and whether a key's page is there."""
        n, page, dim = self.lens_list[b], self.page, self.dim
        at = self.tables[b, :-(-n // page)].long()
        there = ((at >= 0) & (at < self.pages)).repeat_interleave(page)[:n]
        at = at.clamp(0, self.pages - 1)
        both = [torch.ldexp(self.cache[i].view(torch.float8_e4m3fn)[at].double(), (self.scales[i][at].int() - 127).unsqueeze(-1)) for i in range(2)]
        k = both[0].view(-1, self.heads_k, page, dim).transpose(0, 1).reshape(self.heads_k, -1, dim)[:, :n]
        v = both[1].view(-1, self.heads_k, dim, page).permute(1, 0, 3, 2).reshape(self.heads_k, -1, dim)[:, :n]
        return k, v, there


def check_attention(F, c, q, counts, causal, scale=None, out=None, lse=None, first=0, **more):
    heads, tokens, dim = q.shape
    starts = [first]
    for n in counts:
        starts.append(starts[-1] + n)
    mark = 3.0
    out = torch.full((tokens, heads, dim), mark, dtype=torch.bfloat16, device="cuda") if out is None else out
    lse = torch.full((tokens, heads), mark, device="cuda") if lse is None else lse
    scale = dim ** -0.5 if scale is None else scale
    F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints(starts), c.page, scale=scale, causal=causal, out=out, lse=lse, **more)
    group = heads // c.heads_k
    live = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    for b, n in enumerate(counts):
        if n == 0:
            continue
        at = slice(starts[b], starts[b] + n)
        live[at] = True
        k, v, there = (t.repeat_interleave(group, 0) if t.dim() == 3 else t for t in c.values(b))
        x = q[:, at].double()
        keys = torch.arange(k.shape[1], device="cuda")
        hidden = ~there | (keys > (k.shape[1] - n + torch.arange(n, device="cuda")).unsqueeze(1) if causal else torch.zeros(n, 1, dtype=torch.bool, device="cuda"))
        s = torch.matmul(x, k.transpose(1, 2).contiguous()) * scale
        s = s.masked_fill(hidden, -INF)
        top = s.amax(-1, keepdim=True) if s.shape[-1] else torch.full((heads, n, 1), -INF, dtype=torch.float64, device="cuda")
        top = torch.where(top == -INF, 0.0, top)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total == 0, 1.0, total)
        y = torch.matmul(p, v) if s.shape[-1] else torch.zeros(heads, n, dim, dtype=torch.float64, device="cuda")
        # A score: dim products, exact, and as many additions.  A weight: its score's error and its maximum's, the power's argument (twice
        # rounded, up to 8 more than the distance from the maximum in powers of two) and its own rounding, half a bf16 step, in the product.
        off = (dim + 2) * FP32 * scale * torch.matmul(x.abs(), k.abs().transpose(1, 2).contiguous())
        gap = torch.where(hidden, 0.0, (top - s.masked_fill(hidden, 0.0)).abs() / math.log(2) + 8)
        one = torch.where(hidden, 0.0, 2 * off + off.amax(-1, keepdim=True) if s.shape[-1] else off) + gap * 2 * FP32 + 4 * FP32
        adds = (k.shape[1] / 16 + 40) * FP32      # additions one behind the other, of sums and accumulators
        rel = torch.matmul(p, torch.ones(1, device="cuda").double().expand(p.shape[-1], 1)) * 0 + (p * one).sum(-1, keepdim=True) + adds
        tol = torch.matmul(p * (one + BF16 * 1.01), v.abs()) + (rel + BF16 * 1.01) * y.abs() + adds * torch.matmul(p, v.abs()) + 1e-37
        got = out[at].double().transpose(0, 1)
        err = (got - y).abs()
        assert torch.equal(torch.isnan(got), torch.isnan(y))
        bad = (err > tol) & ~torch.isnan(y)
        assert not bad.any(), (b, bad.nonzero()[:3].tolist(), (err - tol)[bad].max().item())
        want = torch.where(total == 0, -INF, top + torch.log(total)).squeeze(-1)
        got = lse[at].double().T
        gone = torch.isinf(want)
        assert torch.equal(gone & (want < 0), torch.isinf(got) & (got < 0))
        err = (got - want).abs()[~gone]
        room = (rel.squeeze(-1) * 1.5 + 8 * FP32 * (want.abs().clamp(max=1e30) + top.squeeze(-1).abs() + 1))[~gone]
        assert (err <= room).all(), (b, (err - room).max().item())
    assert (out[~live] == mark).all() and (lse[~live] == mark).all(), "rows of no sequence"
    return out, lse


@pytest.mark.parametrize("dim", [8, 16, 32, 40, 64, 72, 96, 104, 120, 128])
@pytest.mark.parametrize("page", [16, 128])
def test_attention_channels(F, dim, page):
    c = Paged(F, dim, [200, 65, 1], 2, dim, page)
    q = randn(gen(1), 6, 30, dim).bfloat16()
    check_attention(F, c, q, [1, 1, 1], True)
    check_attention(F, c, q, [17, 9, 1], True)
    check_attention(F, c, q, [20, 3, 7], False)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("heads,heads_k", [(1, 1), (8, 8), (24, 8), (16, 1), (34, 2), (5, 1)])
def test_attention_heads(F, heads, heads_k, page):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300]
    c = Paged(F, heads, lens, heads_k, 64, page)
    q = randn(gen(2), heads, 100, 64).bfloat16()
    check_attention(F, c, q, [1] * len(lens), True, first=5)
    check_attention(F, c, q, [0, 1, 3, 16, 2, 1, 0, 30, 1, 5, 7, 20], True)
    check_attention(F, c, q, [2, 3, 20, 16, 17, 4, 1, 0, 0, 1, 9, 1], False, first=3)   # (more queries than keys, none)
    check_attention(F, c, q, [2, 3, 20, 16, 17, 4, 1, 0, 0, 1, 9, 1], True, first=3)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,counts", [([5000], [1]), ([5000, 3, 700, 2500], [1, 1, 1, 1]), ([3000, 900], [300, 900]), ([20000], [40]), ([6000], [2000]),
                                         ([1] * 100 + [9000], [1] * 101), ([700] * 300, [1] * 300)])
def test_attention_lengths(F, lens, counts, causal):
    """Long and short sequences side by side: keys in parts, tiles of several rows."""
    c = Paged(F, len(lens), lens, 2, 128, 64)
    q = randn(gen(3), 6, sum(counts) + 2, 128).bfloat16()
    check_attention(F, c, q, counts, causal)


def test_attention_of_a_wide_table(F):
    """A table with room for far more than the sequences hold: the same rows as with a narrow one, by other sizes of the launch."""
    lens, counts = [130, 77, 400], [1, 1, 1]
    for wide in (None, 13, 4000):
        c = Paged(F, 5, lens, 4, 72, 32, wide=wide)
        check_attention(F, c, randn(gen(4), 8, 3, 72).bfloat16(), counts, True)


@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("long", [300, 3000])
def test_attention_pages_that_are_none(F, n, long):
    c = Paged(F, 11, [long, 200], 2, 64, 16)
    c.tables[0, 3], c.tables[0, 7], c.tables[0, 10] = -1, c.pages, 2 ** 31 - 1
    c.tables[1, :] = -1                                                     # no key at all
    check_attention(F, c, randn(gen(5), 4, 2 * n, 64).bfloat16(), [n, n], True)
    check_attention(F, c, randn(gen(5), 4, 2 * n, 64).bfloat16(), [n, n], False)


@pytest.mark.parametrize("long", [150, 2000])
def test_attention_values_that_are_no_numbers_stay_behind_a_querys_end(F, long):
    """A NaN in a value (or key) reaches the queries that see it and no other, in tiles of several queries too."""
    for which in (0, 1):
        c = Paged(F, 12, [long], 2, 64, 32)
        place = long - 9
        p = int(c.tables[0, place // 32])
        if which:
            c.cache[1, p].view(2, 64, 32)[1, 5, place % 32] = 0xFF
        else:
            c.cache[0, p].view(2, 32, 64)[1, place % 32, 5] = 0x7F
        q = randn(gen(6), 4, 40, 64).bfloat16()
        out, _ = check_nan_rows(F, c, q, 40, long, place, which)
    q[1, 3, 7] = math.nan
    c = Paged(F, 13, [long], 2, 64, 32)
    out = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, 40]), 32)
    assert out[3, 1].isnan().all() and out.isnan().sum() == 64


def check_nan_rows(F, c, q, n, long, place, which):
    out, lse = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, n]), c.page, want_lse=True)
    sees = torch.arange(long - n, long, device="cuda") >= place
    nan = out.isnan()
    assert not nan[~sees].any() and not nan[:, :2].any() and not lse[~sees].isnan().any()
    if which:
        assert nan[sees][:, 2:, 5].all() and nan[sees].sum() == sees.sum() * 2
        clean = c.cache.clone()
        clean[1, int(c.tables[0, place // 32])].view(2, 64, 32)[1, 5, place % 32] = 0
        ref = F.fb4_cache_attention(q, clean, c.scales, c.tables, c.lens, ints([0, n]), c.page)
        keep = torch.ones(64, dtype=torch.bool, device="cuda")
        keep[5] = False
        assert torch.equal(out[:, :, keep], ref[:, :, keep])   # (channel by channel the same, query by query or not)
        assert torch.equal(out[~sees], ref[~sees])
    else:
        assert nan[sees][:, 2:].all() and lse[sees][:, 2:].isnan().all()
    return out, lse


def test_attention_strides(F):
    heads, tokens, dim = 6, 33, 72
    c = Paged(F, 14, [90, 500], 3, dim, 32)
    packed = randn(gen(7), tokens, 2 * heads, dim).bfloat16()
    q = packed[:, heads:].transpose(0, 1)
    wide = torch.full((tokens, 2, heads, dim + 8), 3.0, dtype=torch.bfloat16, device="cuda")
    out = wide[:, 1, :, :dim]
    check_attention(F, c, q, [20, 10], True, out=out)
    assert (wide[:, 0] == 3).all() and (wide[..., dim:] == 3).all()
    by_head = torch.full((heads, tokens, dim), 3.0, dtype=torch.bfloat16, device="cuda")
    check_attention(F, c, q.contiguous(), [20, 10], False, out=by_head.transpose(0, 1))


@pytest.mark.parametrize("size", [1e-3, 40.0, 3e4])
def test_attention_of_large_scores(F, size):
    c = Paged(F, 15, [600, 4000], 2, 64, 64)
    check_attention(F, c, (randn(gen(8), 4, 40, 64) * size).bfloat16(), [39, 1], True)


def test_attention_scores_without_bounds(F):
    """A score of +Inf: NaN and lse = +Inf; all of them -Inf: zeros and lse = -Inf."""
    for long in (40, 3000):
        c = Paged(F, 16, [long, long], 1, 32, 16)
        c.cache[0, :, :, :] = 0x38                        # keys of 1
        q = torch.ones(1, 2, 32, dtype=torch.bfloat16, device="cuda")
        q[0, 0, 3], q[0, 1, 3] = INF, -INF
        out, lse = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, 1, 2]), 16, want_lse=True)
        assert out[0].isnan().all() and lse[0, 0] == INF and (out[1] == 0).all() and lse[1, 0] == -INF


def test_attention_of_no_sequence(F):
    c = Paged(F, 17, [], 2, 64, 16)
    q = randn(gen(9), 2, 5, 64).bfloat16()
    out = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0]), 16)
    assert (out == 0).all()
    c = Paged(F, 17, [0, 0], 2, 64, 16, spare=0)
    out, lse = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, 2, 4]), 16, want_lse=True)
    assert (out == 0).all() and (lse[:4] == -INF).all() and (lse[4] == 0).all()


def test_starts_and_lengths_that_are_none_stay_in_bounds(F):
    """Rows past the tensor, falling starts, lengths past the table: clamped, nothing else written."""
    c = Paged(F, 18, [100, 100, 100], 2, 64, 16)
    q = randn(gen(10), 2, 6, 64).bfloat16()
    for long in (2 ** 31 - 1, -5, 100):
        c.lens[:] = long
        for starts in ([0, 2, 4, 9], [-3, 2, 1, 6], [5, 5, 2 ** 31 - 1, 6], [6, 4, 2, 0], [-2 ** 31] * 4):
            for causal in (True, False):
                F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints(starts), 16, causal=causal)
    torch.cuda.synchronize()


def test_offsets_beyond_32_bits(F):
    """Pages behind 4 GiB of keys, and the values' half behind 8."""
    heads_k, dim, page = 8, 128, 64
    pages = (5 << 30) // (heads_k * dim * page)
    cache = torch.empty(2, pages, heads_k, page * dim, dtype=torch.uint8, device="cuda")
    scales = torch.empty(2, pages, heads_k, dtype=torch.uint8, device="cuda")
    small = Paged(F, 19, [200, 90], heads_k, dim, page)
    far = [pages - 1 - 3 * i for i in range(small.pages)]
    cache[:, far], scales[:, far] = small.cache, small.scales
    q = randn(gen(11), 16, 8, dim).bfloat16()
    starts = ints([0, 5, 8])
    want = F.fb4_cache_attention(q, small.cache, small.scales, small.tables, small.lens, starts, page)
    tables = torch.where(small.tables >= 0, pages - 1 - 3 * small.tables, -1)
    assert torch.equal(F.fb4_cache_attention(q, cache, scales, tables.contiguous(), small.lens, starts, page), want)
    k, v = randn(gen(12), heads_k, 70, dim).bfloat16(), randn(gen(13), heads_k, 70, dim).bfloat16()
    at = torch.arange(30, 100, device="cuda", dtype=torch.int32)
    F.fb4_cache_store(k, v, at + small.page * 1, small.cache, small.scales, page)
    place = at + small.page
    F.fb4_cache_store(k, v, ((pages - 1 - 3 * (place // page)) * page + place % page).int(), cache, scales, page)
    assert torch.equal(cache[:, far], small.cache) and torch.equal(scales[:, far], small.scales)


# ------------------------------------------------------------------------------------------------ together
class Served:
    """A layer's serving state, and its step: products, plan, norm and rotation, store, attention, product."""

    def __init__(self, F, luts, seed, batch=5, heads=6, heads_k=2, dim=64, page=16, wide=40):
        g = gen(seed)
        self.F, self.luts, self.heads, self.heads_k, self.dim, self.page = F, luts, heads, heads_k, dim, page
        self.width = heads * dim
        self.qkv = weights(F, luts, g, (heads + 2 * heads_k) * dim, self.width, 32, self.width ** -0.5)
        self.proj = weights(F, luts, g, self.width, self.width, 32, self.width ** -0.5)
        self.freqs = 100.0 ** (-torch.arange(dim // 2, dtype=torch.float64, device="cuda") / (dim // 2))
        pages = batch * wide
        self.cache = torch.zeros(2, pages, heads_k, page * dim, dtype=torch.uint8, device="cuda")
        self.scales = torch.zeros(2, pages, heads_k, dtype=torch.uint8, device="cuda")
        self.tables = torch.full((batch, wide), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, device="cuda", generator=g).int()
        self.count, self.lens = ints([pages]), torch.zeros(batch, dtype=torch.int32, device="cuda")

    def step(self, x, adds, stream=None):
        F, n = self.F, x.shape[0]
        qkv = F.fb4_matvec(self.luts, x, *self.qkv, stream=stream).view(1, n, -1, self.dim).transpose(1, 2)
        h, hk = self.heads, self.heads_k
        _, _, starts, slots, positions = F.fb4_cache_plan(self.lens, adds, self.tables, self.free, self.count, self.page, n, lens_out=self.lens,
                                                          free_count_out=self.count, stream=stream)
        q, k = F.fb4_qk_norm_rope(qkv[:, :h], qkv[:, h:h + hk], positions.view(1, n, 1), self.freqs, (self.dim // 2,), stream=stream)
        F.fb4_cache_store(k[0], qkv[0, h + hk:], slots, self.cache, self.scales, self.page, stream=stream)
        a = F.fb4_cache_attention(q[0], self.cache, self.scales, self.tables, self.lens, starts, self.page, stream=stream)
        y = F.fb4_matvec(self.luts, a.view(n, -1), *self.proj, stream=stream)
        return a, y, q, k, qkv


def test_a_prompt_at_once_or_token_by_token(F, luts):
    """A sequence's last output from the whole prompt and from its tokens one by one differ by the roundings of what the cache holds:
    the scales grow while tokens come, and elements below a page's largest by 2^14 and more lose bits then."""
    n, other = 37, Served(F, luts, 21, batch=1)
    x = randn(gen(22), n, other.width).bfloat16()
    a_all, _, q, k, qkv = other.step(x, ints([n]))
    # against float64, by the keys and values before they were stored: E4M3 is off by at most 2^-4 of an element
    kk, vv = k[0].double(), qkv[0, other.heads + other.heads_k:].double()
    one = Served(F, luts, 21, batch=1)
    rows = torch.cat([one.step(x[i:i + 1], ints([1]))[0] for i in range(n)])
    assert one.lens.item() == other.lens.item() == n and torch.equal(one.tables, other.tables)
    group = other.heads // other.heads_k
    s = torch.matmul(q[0].double(), kk.repeat_interleave(group, 0).transpose(1, 2).contiguous()) * other.dim ** -0.5
    hidden = torch.arange(n, device="cuda") > torch.arange(n, device="cuda").unsqueeze(1)
    size = torch.matmul(q[0].double().abs(), kk.abs().repeat_interleave(group, 0).transpose(1, 2).contiguous()) * other.dim ** -0.5
    p = torch.softmax(s.masked_fill(hidden, -INF), -1)
    y = torch.matmul(p, vv.repeat_interleave(group, 0))
    worst = torch.where(hidden, 0.0, size).amax(-1, keepdim=True) * 2.0 ** -4      # of a score
    spread = torch.exp(2 * worst) - 1
    tol = (spread + 2.0 ** -4 * (1 + spread) + 4 * BF16) * torch.matmul(p, vv.abs().repeat_interleave(group, 0)) + 1e-4
    for got in (a_all, rows):
        assert ((got.double().transpose(0, 1) - y).abs() <= tol).all()


def run_steps(F, luts, steps, stream=None):
    state = Served(F, luts, 30)
    g = gen(31)
    outs = []
    for i in range(steps):
        adds = [[3, 9, 1, 20, 0], [1, 1, 1, 1, 1], [1, -4, 1, 1, 5]][i % 3]
        x = randn(g, 40, state.width).bfloat16()
        outs.append(state.step(x, ints(adds), stream)[1].clone())
    return outs, state


def test_steps_on_another_stream(F, luts):
    want, _ = run_steps(F, luts, 6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = run_steps(F, luts, 6)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_captured_step_is_replayed_with_other_lengths(F, luts):
    """One graph for every step: the launches do not depend on what the lengths, tables and counts hold."""
    want, end = run_steps(F, luts, 9)
    state = Served(F, luts, 30)
    g = gen(31)
    x = torch.zeros(40, state.width, dtype=torch.bfloat16, device="cuda")
    adds = torch.zeros(5, dtype=torch.int32, device="cuda")
    state.step(x, adds)                       # (the memory it needs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = state.step(x, adds)[1]
    for i in range(9):
        adds.copy_(ints([[3, 9, 1, 20, 0], [1, 1, 1, 1, 1], [1, -4, 1, 1, 5]][i % 3]))
        x.copy_(randn(g, 40, state.width).bfloat16())
        graph.replay()
        if i % 3 == 2:
            torch.cuda.synchronize()
        assert torch.equal(y, want[i]), i
    for name in ("cache", "scales", "tables", "lens", "count", "free"):
        assert torch.equal(getattr(state, name), getattr(end, name)), name


def test_given_workspaces(F):
    c = Paged(F, 23, [5000], 2, 64, 64)
    q = randn(gen(24), 4, 3, 64).bfloat16()
    need = F.binding.lib().fb4_cache_attention_workspace(3, 4, 2, 64, 64, c.tables.shape[1], 1)
    assert need > 0
    want = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, 3]), 64)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    got = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, 3]), 64, workspace=ws[:need])
    assert torch.equal(got, want) and (ws[need:] == 0xFF).all()
    for bad, code in ((ws[:need - 1], F.ERR_INVALID_ARG), (ws[4:need + 4], F.ERR_UNSUPPORTED)):
        with pytest.raises(F.Fb4Error) as e:
            F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, 3]), 64, workspace=bad)
        assert e.value.code == code


def test_both_bindings_answer_alike(F, luts, monkeypatch):
    B = F.binding
    if B._call is B.CtypesCall:
        pytest.skip("no C module for this interpreter")
    monkeypatch.setattr(B, "_serving_call", B.ServingCall)
    ctypes_outs, ctypes_state = run_steps(F, luts, 4)
    ws_outs = ctypes_state.step(randn(gen(1), 1, ctypes_state.width).bfloat16(), ints([1, 0, 0, 0, 0]))[0]
    asked = []

    class Noted:
        def __getattr__(self, name):
            def call(*a):
                asked.append(name)
                raise AssertionError("handed over: " + name)
            return call
    monkeypatch.setattr(B, "_serving_call", B._call)
    B._call.bind_serving(type("Elsewhere", (), {n: staticmethod(getattr(Noted(), n)) for n in ("matvec", "cache_plan", "cache_store", "cache_attention")}))
    try:
        outs, state = run_steps(F, luts, 4)
        rows = state.step(randn(gen(1), 1, state.width).bfloat16(), ints([1, 0, 0, 0, 0]))[0]
    finally:
        B._call.bind_serving(B.ServingCall)
    assert not asked and all(torch.equal(a, b) for a, b in zip(outs, ctypes_outs)) and torch.equal(rows, ws_outs)
    assert torch.equal(state.cache, ctypes_state.cache)
    # what the module does not take is refused by the same rules
    x = randn(gen(1), 2, state.width).bfloat16()
    for bad in (lambda: F.fb4_matvec(luts, x.float(), *state.qkv), lambda: F.fb4_matvec(luts, x.cpu(), *state.qkv), lambda: F.fb4_matvec(luts, x, *state.qkv, block=16),
                lambda: F.fb4_matvec(luts, x[:, ::2], *state.qkv), lambda: F.fb4_matvec(luts, x, *state.qkv, block=2 ** 32 + 32),
                lambda: F.fb4_cache_plan(state.lens, state.lens[:2], state.tables, state.free, state.count, 16, 4),
                lambda: F.fb4_cache_plan(state.lens, state.lens, state.tables, state.free, state.count, 2 ** 32 + 16, 4),
                lambda: F.fb4_cache_plan(state.lens, state.lens, state.tables.t(), state.free, state.count, 16, 4),
                lambda: F.fb4_cache_plan(state.lens, state.lens, state.tables, state.free, state.count, 24, 4),
                lambda: F.fb4_cache_store(x.view(2, -1, 64), x.view(2, -1, 64), state.lens, state.cache, state.scales, 16),
                lambda: F.fb4_cache_attention(x.view(2, -1, 64), state.cache, state.scales, state.tables, state.lens, state.lens, 16)):
        with pytest.raises(F.Fb4Error):
            bad()


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("rows,n,cols", [(1, 16500, 40032), (3, 8250, 33344), (40, 4100, 33024), (33, 5000, 1088), (18, 16400, 20000), (2, 300, 33568), (2, 100, 65600)])
def test_products_of_many_channels(F, luts, rows, n, cols, block):
    """More channels than a workgroup holds scales of at a time; words that lie 16 bytes apart and not."""
    g = gen(rows + n)
    codes = torch.randint(0, 256, (n, cols // 2), device="cuda", generator=g, dtype=torch.uint8)
    meta = torch.randint(120, 125, (n, cols // block), device="cuda", generator=g, dtype=torch.int16) * 256 + torch.randint(0, 32, (n, cols // block), device="cuda", generator=g, dtype=torch.int16)
    x = randn(g, rows, cols).bfloat16()
    check_product(F, luts, x, codes, meta, block, None, F.fb4_matvec(luts, x, codes, meta, block=block, out_dtype=F.DTYPE_F32))
    # words that begin at any multiple of their size
    at = torch.empty(meta.numel() + 8, device="cuda", dtype=torch.int16)
    shift = 2 if block == 16 else 1
    at[shift:shift + meta.numel()] = meta.view(-1)
    x = randn(g, rows, cols).bfloat16()
    same = F.fb4_matvec(luts, x, codes, meta, block=block)
    assert torch.equal(same, F.fb4_matvec(luts, x, codes, at[shift:shift + meta.numel()].view(meta.shape), block=block))


# (whether sums are relative to a rounded or an exact product changes at 2^20 powers of two)
@pytest.mark.parametrize("n,long", [(1, 700), (3, 4000), (60, 700), (60, 5000)])
@pytest.mark.parametrize("first,later,scale", [(1.0, 3e4, 1.0), (3e4, 1.0, 1.0), (-3e4, 3e4, 1.0), (3e4, 3e4, 2.0 ** 20), (3e4, -3e4, 2.0 ** 40), (1.0, 1.5, 2.0 ** 18), (1e-3, 1.0, 1e-30)])
def test_attention_scores_that_rise_by_far(F, n, long, first, later, scale):
    """Keys of one size and then of another: the maximum moves within a wavefront's walk, between wavefronts and between parts.  Scores are
    products of few numbers, whose sums are exact in fp32, so that a weight far below its row's largest is nothing in both."""
    c = Paged(F, 31, [long], 2, 16, 16, scale_spread=1)
    held = c.tables[0, :-(-long // 16)].long()
    keys = torch.zeros(held.numel() * 16, 16, device="cuda")
    keys[:, 0] = torch.where(torch.arange(keys.shape[0], device="cuda") < long // 2, first, later)
    keys[::7, 0] *= 0.5
    sizes = torch.ldexp(torch.ones((), device="cuda"), torch.ceil(torch.log2(keys.abs().amax() / 448)).int())
    c.cache[0, held] = (keys / sizes).to(torch.float8_e4m3fn).view(torch.uint8).view(-1, 1, 256).expand(-1, 2, -1).contiguous()
    c.scales[0] = int(torch.log2(sizes).item()) + 127
    q = torch.zeros(4, n, 16, device="cuda", dtype=torch.bfloat16)
    q[..., 0] = (torch.arange(4 * n, device="cuda").view(4, n) % 5 - 2).bfloat16()
    check_attention(F, c, q, [n], True, scale=scale)


@pytest.mark.parametrize("n,group", [(32, 1), (100, 1), (10, 3)])
def test_attention_rows_of_far_larger_scores_beside_others(F, n, group):
    """Sixteen rows' scores pass 2^20 powers of two half way; their neighbours' weights stay what they are, with a maximum whose product
    with the scale does not fit fp32."""
    long, dim = 1400, 16
    c = Paged(F, 37, [long], 1, dim, 16, scale_spread=1)
    held = c.tables[0, :-(-long // 16)].long()
    keys = torch.zeros(held.numel() * 16, dim, device="cuda")
    at = torch.arange(keys.shape[0], device="cuda")
    keys[:, 0] = torch.where(at < long // 2, 2.0 ** -5, 448.0)
    keys[:, 1] = 416.0
    c.cache[0, held] = keys.to(torch.float8_e4m3fn).view(torch.uint8).view(-1, 1, 16 * dim)
    c.scales[0] = 127
    q = torch.zeros(group, n, dim, device="cuda", dtype=torch.bfloat16)
    # (token by token, the heads of a key head side by side: sixteen rows after sixteen)
    second = (torch.arange(n, device="cuda") * group + torch.arange(group, device="cuda").unsqueeze(1)) // 16 % 2 == 1
    q[..., 0], q[..., 1] = torch.where(second, 0.0, 4096.0).bfloat16(), torch.where(second, 1237.0, 0.0).bfloat16()
    check_attention(F, c, q, [n], True, scale=0.7)
    out, lse = check_attention(F, c, q, [n], False, scale=1.0)
    q[~second] = 0
    alone, lse_alone = check_attention(F, c, q, [n], False, scale=1.0)
    assert torch.equal(out[second.T], alone[second.T]) and torch.equal(lse[second.T], lse_alone[second.T])


@pytest.mark.parametrize("long,n", [(150, 3), (150, 8), (2000, 3), (2000, 20)])
def test_attention_nan_values_in_tiles_of_few_rows(F, long, n):
    """As above for tiles of 16 and 32 rows: a NaN among the last keys, seen by some of the queries."""
    for place in (long - 2, long - n, long - n - 1):
        c = Paged(F, 41, [long], 2, 64, 32)
        c.cache[1, int(c.tables[0, place // 32])].view(2, 64, 32)[1, 5, place % 32] = 0x7F
        q = randn(gen(42), 4, n, 64).bfloat16()
        check_nan_rows(F, c, q, n, long, place, 1)


def test_attention_pages_that_are_none_beside_nan(F):
    """A missing page's keys are skipped; a NaN in the same 64 keys is seen by those who see its key."""
    for n in (3, 40):
        c = Paged(F, 43, [600], 1, 64, 16)
        c.tables[0, 5] = -1
        c.cache[1, int(c.tables[0, 6])].view(64, 16)[7, 3] = 0xFF
        q = randn(gen(44), 2, n, 64).bfloat16()
        check_attention(F, c, q, [n], True)
        out = F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, n]), 16)
        assert out[:, :, 7].isnan().all() and out.isnan().sum() == 2 * n


def test_prompts_and_single_tokens_in_one_call(F):
    """What a server sends: sequences at their prompts beside others a token further, some idle, rows left over."""
    lens = [900, 1, 4000, 300, 77, 0, 2500, 640]
    counts = [900, 1, 1, 120, 1, 0, 333, 1]
    for heads, heads_k, dim, page in ((24, 8, 128, 64), (16, 16, 72, 16), (4, 2, 40, 128)):
        c = Paged(F, 45, lens, heads_k, dim, page)
        q = randn(gen(46), heads, sum(counts) + 9, dim).bfloat16()
        check_attention(F, c, q, counts, True, first=4)
        check_attention(F, c, q, counts, False, first=4)


def test_plans_without_positions_and_many_sequences(F):
    r = random.Random(3)
    lens = [r.randint(0, 200) for _ in range(1500)]
    adds = [r.choice([1, 0, 17, 40, -3, -500]) for _ in range(1500)]
    ids = list(range(1500 * 16))
    tables = [[ids.pop() if p * 16 < lens[b] else -1 for p in range(16)] for b in range(1500)]
    want = check_plan(F, lens, adds, tables, ids, len(ids), 16, sum(max(a, 0) for a in adds))
    t = [ints(x) for x in (lens, adds, tables, ids, [len(ids)])]
    tokens = len(want["slots"])
    out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (1500, 1, 1501, tokens)]
    import ctypes
    P = lambda x: ctypes.c_void_p(x.data_ptr())
    rc = F.binding.lib().fb4_cache_plan(P(t[0]), P(t[1]), 1500, 16, P(t[2]), 16, P(t[3]), len(ids), P(t[4]), P(out[0]), P(out[1]), P(out[2]), P(out[3]), None, tokens,
                                        torch.cuda.current_stream().cuda_stream)
    assert rc == F.OK and [x.cpu().tolist() for x in out] == [want["lens"], want["count"], want["starts"], want["slots"]]


def test_two_calls_at_once_on_two_streams(F):
    """Each with its own workspace: the results are those of one after the other."""
    c, d = Paged(F, 47, [5000, 300], 2, 64, 64), Paged(F, 48, [7000, 3000], 2, 64, 64)
    q = randn(gen(49), 4, 2, 64).bfloat16()
    starts = ints([0, 1, 2])
    want = [F.fb4_cache_attention(q, x.cache, x.scales, x.tables, x.lens, starts, 64) for x in (c, d)]
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        got += [F.fb4_cache_attention(q, x.cache, x.scales, x.tables, x.lens, starts, 64, stream=s) for x, s in ((c, a), (d, b))]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 2]) for i, g in enumerate(got))


@pytest.mark.parametrize("dim", [72, 128])
@pytest.mark.parametrize("counts", [[1, 1, 1, 1, 0], [6, 1, 6, 2, 3], [150, 150, 150, 150, 1], [1, 500, 40, 1, 0]])
def test_attention_of_one_part_beside_several(F, counts, dim):
    """Short and long sequences in a call: a tile of one part writes its rows itself, the others' parts meet.  Nothing of what the workspace held counts."""
    lens = [200, 9000, 600, 3000, 7]
    c = Paged(F, 51, lens, 2, dim, 64)
    q = randn(gen(52), 6, sum(counts) + 5, dim).bfloat16()
    for causal in (True, False):
        size = F.binding.lib().fb4_cache_attention_workspace(q.shape[1], 6, 2, dim, 64, c.tables.shape[1], len(lens))
        assert size > 0
        work = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
        check_attention(F, c, q, counts, causal, first=2, workspace=work)


@pytest.mark.parametrize("block", [32, 16])
@pytest.mark.parametrize("rows,n,cols", [(1, 33000, 64), (4, 12300, 160), (5, 4100, 96), (8, 32770, 32), (9, 8200, 352), (16, 8193, 1184), (32, 9000, 64), (64, 4097, 96)])
def test_products_of_many_rows_of_weights(F, luts, rows, n, cols, block):
    """Several tiles of the weights to a workgroup, by their number and that of the rows; the last ones ragged."""
    g = gen(rows + n + cols + block)
    codes, meta = weights(F, luts, g, n, cols, block)
    x, bias = randn(g, rows, cols).bfloat16(), randn(g, n)
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full((rows, n), 7.0, dtype=dtype, device="cuda")
        F.fb4_matvec(luts, x, codes, meta, block, bias, out=out)
        check_product(F, luts, x, codes, meta, block, bias, out)


def test_one_prompt_among_many_single_tokens(F):
    lens = [9 + b % 50 for b in range(499)] + [6000]
    c = Paged(F, 53, lens, 1, 64, 64)
    q = randn(gen(54), 3, 499 + 6000, 64).bfloat16()
    check_attention(F, c, q, [1] * 499 + [6000], True)


# (growths of the scale's byte on which its inverse is a normal number, 0, and past all exponents)
@pytest.mark.parametrize("old", [0, 10, 19, 110])
def test_stores_whose_scale_grows_by_far(F, old):
    """What a page holds is rounded to a scale that is larger by up to 2^247: beyond 2^18 everything is below half of E4M3's least number."""
    page, dim, heads = 16, 16, 2
    growths = [n for n in (1, 5, 17, 18, 19, 100, 126, 127, 128, 129, 130, 200, 237, 247) if 10 <= old + n <= 247]
    for tokens in (1, 6):
        g = gen(old + tokens)
        cache, scales = new_cache(g, len(growths), heads, dim, page)
        cache[:, :, 0] = 0                          # a head of zeros, one of anything, a NaN in it
        cache[:, :, 1, 15 * 16 + 15] = 0x7F
        scales[:] = old
        x = torch.zeros(heads, len(growths) * tokens, dim)
        for i, n in enumerate(growths):             # 160 and -240 times the new scale
            x[:, i * tokens:(i + 1) * tokens] = 1.25 * 2.0 ** (old + n - 120)
            x[:, (i + 1) * tokens - 1, 3] *= -1.5
        x = x.bfloat16().cuda()
        at = [i * page + 3 + t for i in range(len(growths)) for t in range(tokens)]
        check_store(F, x, x.flip(2), at, cache, scales, page)
        assert (scales.cpu() == torch.tensor([old + n for n in growths]).view(1, -1, 1)).all()


@pytest.mark.parametrize("begin", [0.0, 2.0 ** -100])
def test_stores_of_large_tokens_behind_small_ones(F, begin):
    """A page that a token of zeros (or next to nothing) begins, and one from 5e5 to 3e38 behind it, singly and as runs."""
    page, dim, heads, sizes = 32, 24, 2, (4.6e5, 5e5, 9e5, 1e6, 2.0 ** 60, 3e38)
    for tokens in (1, 5):
        cache, scales = torch.zeros(2, len(sizes), heads, page * dim, dtype=torch.uint8, device="cuda"), torch.zeros(2, len(sizes), heads, dtype=torch.uint8, device="cuda")
        first = torch.full((heads, len(sizes), dim), begin).bfloat16().cuda()
        first[:, :, 5] *= -1
        check_store(F, first, first, [p * page for p in range(len(sizes))], cache, scales, page)
        x = randn(gen(60), heads, len(sizes) * tokens, dim)
        x = x / x.abs().amax((0, 2), keepdim=True) * torch.tensor(sizes, device="cuda").repeat_interleave(tokens).view(1, -1, 1)
        at = [p * page + 1 + t for p in range(len(sizes)) for t in range(tokens)]
        check_store(F, x.bfloat16(), x.flip(2).bfloat16(), at, cache, scales, page)
        assert np.isfinite(values_of(cache)).all()


@pytest.mark.parametrize("tile", [16, 128])
@pytest.mark.parametrize("heads,heads_k", [(1, 1), (3, 1), (6, 2), (2, 2)])
@pytest.mark.parametrize("first", [1, 3])
def test_attention_in_parts_behind_rows_of_no_sequence(F, heads, heads_k, first, tile):
    """A wavefront that joins rows has some of no sequence and then some of the first one, whose keys are in several parts."""
    if tile == 16:   # (at most 40 rows to a sequence)
        lens = [5000] + [300 + 7 * b for b in range(43)]
        counts = [30 * heads_k // heads] + [25 * heads_k // heads] * 43
    else:
        lens, counts = [9000, 700], [900, 300]
    c = Paged(F, 61, lens, heads_k, 64, 64)
    tokens = first + sum(counts) + 2
    assert tokens * heads > 1024 and heads * first % 4
    assert F.binding.lib().fb4_cache_attention_workspace(tokens, heads, heads_k, 64, 64, c.tables.shape[1], len(lens)) > 0
    q = randn(gen(62), heads, tokens, 64).bfloat16()
    for causal in (True, False):
        check_attention(F, c, q, counts, causal, first=first)


@pytest.mark.parametrize("long,n", [(150, 3), (150, 40), (2000, 3), (2000, 40), (130, 9), (130, 70)])
@pytest.mark.parametrize("dim", [64, 72])
@pytest.mark.parametrize("element", [0x78, 0xF8, 0x7E])
def test_attention_values_past_the_largest_number_stay_behind_a_querys_end(F, long, n, dim, element):
    """An element that the largest scale takes to 2^128 and beyond is Inf as an operand, whose product with a weight of 0 is no number."""
    for place in (long - 2, long - n, long - n - 1):
        c = Paged(F, 63, [long], 2, dim, 32)
        p = int(c.tables[0, place // 32])
        held = c.cache[1, p].view(2, dim, 32)[1]
        held[:, :] = 0
        c.scales[1, p, 1] = 247
        if long % 32 and p == int(c.tables[0, long // 32]):
            held[:, long % 32:] = 0x7E           # (past all numbers as well, behind the sequence's end)
        q = randn(gen(64), 4, n, dim).bfloat16()
        call = lambda: F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints([0, n]), c.page)
        want = call()
        assert want[:, :2].isfinite().all()
        held[5, place % 32] = element
        out = call()
        sees = torch.arange(long - n, long, device="cuda") >= place
        assert torch.equal(out[~sees], want[~sees]) and want[~sees].isfinite().all()
        assert not out[sees][:, 2:, 5].isfinite().any()
        keep = torch.ones(dim, dtype=torch.bool, device="cuda")
        keep[5] = False
        assert torch.equal(out[:, :, keep], want[:, :, keep]) and torch.equal(out[:, :2], want[:, :2])


def test_the_largest_numbers_through_the_cache(F):
    """A stored magnitude from 1.9375 * 2^127 on is held as 2^128; queries that do not see it are as without it, and keep their numbers."""
    page, dim, n, large = 16, 16, 40, 3.3895313892515355e38
    k, v = randn(gen(65), 1, n, dim).bfloat16(), randn(gen(66), 1, n, dim).bfloat16()
    q = randn(gen(67), 2, n, dim).bfloat16()
    outs = []
    for x in (0.0, large, -large, 1.875 * 2.0 ** 127):
        v[0, 33, 7] = x
        cache, scales = torch.zeros(2, 3, 1, page * dim, dtype=torch.uint8, device="cuda"), torch.zeros(2, 3, 1, dtype=torch.uint8, device="cuda")
        check_store(F, k, v, list(range(n)), cache, scales, page)
        outs.append(F.fb4_cache_attention(q, cache, scales, ints([[0, 1, 2]]), ints([n]), ints([0, n]), page))
    assert all(o[:33].isfinite().all() for o in outs) and not any(o[33:, :, 7].isfinite().any() for o in outs[1:3]) and outs[3].isfinite().all()
    assert all(torch.equal(o[:32], outs[0][:32]) for o in outs)      # (keys 32 .. share a page, whose scale is another then)
    assert all(torch.equal(o[32], outs[3][32]) for o in outs[1:3])


@pytest.mark.parametrize("heads,heads_k,tokens,wide,batch", [(2, 2, 6, 9, 3), (2, 2, 6, 600, 3), (3, 1, 500, 600, 3), (3, 1, 500, 600, 48), (6, 2, 400, 9, 3)])
def test_nothing_is_written_beside_what_starts_and_lengths_name(F, heads, heads_k, tokens, wide, batch):
    """Rows past the tensor, falling starts, lengths past the table, between marked margins: whole calls and ones in parts, joined by one
    wavefront to a row and by several.  What is ascending after clamping is compared with float64."""
    dim, page, mark, margin = 64, 16, 3.0, 4096
    long = 100 if wide < 64 else 3000
    c = Paged(F, 68, [long] * batch, heads_k, dim, page, wide=wide)
    q = randn(gen(69), heads, tokens, dim).bfloat16()
    size = F.binding.lib().fb4_cache_attention_workspace(tokens, heads, heads_k, dim, page, wide, batch)
    assert (size > 0) == (wide > 64)
    few = tokens // 2
    spread = [i * few // batch for i in range(batch)]
    for starts in (spread + [few + 1], spread + [10 ** 6], [-5] + spread[1:] + [few], [few] * batch + [2 ** 31 - 1], [(-1) ** i * i * tokens for i in range(batch + 1)],
                   [tokens - i for i in range(batch + 1)], [tokens if i % 2 else 0 for i in range(batch + 1)], [-2 ** 31] * (batch + 1), [2 ** 31 - 1] * (batch + 1)):
        at = [min(max(s, 0), tokens) for s in starts]
        for n_keys in (long, 2 ** 31 - 1, -5):
            c.lens[:] = n_keys
            for causal in (True, False):
                n = tokens * heads * dim
                memory, sums = torch.full((n + 2 * margin,), mark, dtype=torch.bfloat16, device="cuda"), torch.full((tokens * heads + 2 * margin,), mark, device="cuda")
                out, lse = memory[margin:margin + n].view(tokens, heads, dim), sums[margin:margin + tokens * heads].view(tokens, heads)
                work = torch.full((size + 2 * margin,), 0xA5, dtype=torch.uint8, device="cuda")
                F.fb4_cache_attention(q, c.cache, c.scales, c.tables, c.lens, ints(starts), page, causal=causal, out=out, lse=lse, workspace=work[margin:margin + size] if size else None)
                for t in (memory, sums):
                    assert (t[:margin] == mark).all() and (t[-margin:] == mark).all()
                assert (work[:margin] == 0xA5).all() and (work[margin + size:] == 0xA5).all()
                named = torch.zeros(tokens, dtype=torch.bool, device="cuda")
                for a, b in zip(at, at[1:]):
                    named[a:b] = True
                assert (out[~named] == mark).all() and (lse[~named] == mark).all()
                if at == sorted(at) and n_keys == long:
                    counts = [b - a for a, b in zip(at, at[1:])]
                    got, got_lse = check_attention(F, c, q, counts, causal, first=at[0])
                    assert torch.equal(got, out) and torch.equal(got_lse, lse)


def test_products_into_the_memory_beside_x(F, luts):
    """Results between the rows of x in one buffer are served; on a row of x they are refused and nothing is written."""
    g = gen(70)
    codes, meta = weights(F, luts, g, 96, 256, 32)
    held = randn(g, 9, 512).bfloat16()
    x, want = held[:, :256], F.fb4_matvec(luts, held[:, :256], codes, meta)
    kept = held.clone()
    for first in (250, 0, 160):
        with pytest.raises(F.Fb4Error) as e:
            F.fb4_matvec(luts, x, codes, meta, out=held[:, first:first + 96])
        assert e.value.code == F.ERR_INVALID_ARG and torch.equal(held, kept)
    F.fb4_matvec(luts, x, codes, meta, out=held[:, 256:352])
    assert torch.equal(held[:, 256:352], want) and torch.equal(x, kept[:, :256]) and torch.equal(held[:, 352:], kept[:, 352:])


def test_products_of_no_channels(F, luts):
    """Of empty tensors as torch makes them: the bias, or zeros."""
    none = lambda *shape, t=torch.bfloat16: torch.empty(*shape, 0, dtype=t, device="cuda")
    bias = randn(gen(71), 33)
    for rows in (1, 4, 64):
        for b, want in ((bias, bias), (None, torch.zeros(33, device="cuda"))):
            assert torch.equal(F.fb4_matvec(luts, none(rows), none(33, t=torch.uint8), none(33, t=torch.int16), bias=b, out_dtype=F.DTYPE_F32), want.expand(rows, 33))
