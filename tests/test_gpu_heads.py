"""The attention path against its definitions in 64 bits: norm and rotation of queries and keys, the choice of key blocks,
attention over listed blocks.  A rounding to bf16 is off by at most 2^-8 of the value, one to fp32 by 2^-24."""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, TINY = 2.0 ** -8, 2.0 ** -126   # (a subnormal may come out as zero)


@pytest.fixture(scope="module")
def F():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2603_02883_amd as F
    return F


def agree(got, ref, bound, where=None):
    """Within the bound, or the same infinity, or NaN on both sides (where `where`)."""
    same = ((got - ref).abs() <= bound) | (got == ref) | (got.isnan() & ref.isnan())
    return bool((same if where is None else same | ~where).all())


def rand(*shape, seed=0, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + sum(shape))
    return (torch.randn(*shape, device="cuda", generator=g) * scale).bfloat16()


# ------------------------------------------------------------------------------------------------ norm and rotation
def rope_reference(x, positions, freqs, axis_pairs, gamma, eps, norm, halves):
    """(result, |u| + |w| of each channel's pair) in 64 bits."""
    y = x.double()
    if norm:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
        if gamma is not None:
            y = y * gamma.double()
    out, mass, at, pairs = y.clone(), y.abs(), 0, sum(axis_pairs)
    for a, n in enumerate(axis_pairs):
        t = positions[:, :, a].double()[:, None, :, None] * freqs[at:at + n]
        for j in range(n):
            u, w = (at + j, pairs + at + j) if halves else (2 * (at + j), 2 * (at + j) + 1)
            cos, sin = t[..., j].cos(), t[..., j].sin()
            out[..., u], out[..., w] = y[..., u] * cos - y[..., w] * sin, y[..., u] * sin + y[..., w] * cos
            mass[..., u] = mass[..., w] = y[..., u].abs() + y[..., w].abs()
        at += n
    return out, mass


def check_rope(F, q, k, axis_pairs, positions, gammas=(None, None), eps=1e-6, norm=True, halves=False):
    n = len(axis_pairs)
    freqs = torch.cat([10000.0 ** (-torch.arange(p, dtype=torch.float64, device="cuda") / p) for p in axis_pairs]) if n else None
    guard = 64
    outs = []
    for x in (q, k):
        flat = torch.full((x.numel() + 2 * guard,), -7.0, device="cuda", dtype=torch.bfloat16) if x is not None else None
        outs.append((flat, flat[guard:-guard].view(x.shape)) if x is not None else (None, None))
    got = F.fb4_qk_norm_rope(q, k, positions, freqs, axis_pairs, gamma_q=gammas[0], gamma_k=gammas[1], eps=eps, norm=norm,
                             pairing=F.ROPE_HALVES if halves else F.ROPE_ADJACENT, q_out=outs[0][1], k_out=outs[1][1])
    torch.cuda.synchronize()
    for x, gamma, (flat, out), y in zip((q, k), gammas, outs, got):
        if x is None:
            assert y is None
            continue
        assert y is out and (flat[:guard] == -7.0).all() and (flat[-guard:] == -7.0).all()
        ref, mass = rope_reference(x, positions if n else torch.zeros(1, x.shape[2], 0), freqs, axis_pairs, gamma, eps, norm, halves)
        # the norm in fp32: dim + 16 roundings under a root, then rsqrt and the products; sine and cosine are 2^-22 off at most
        bound = (BF16 * ref.abs() + mass * 2.0 ** -16) * (1 + BF16) + TINY
        right = agree(out.double(), ref, bound)
        assert right, (x.shape, axis_pairs, norm, halves)


ROPES = [
    # batch, tokens, heads_q, heads_k, dim, axis pairs, halves
    (1, 1, 1, 1, 8, (1,), False), (1, 1, 24, 24, 128, (16, 24, 24), False), (2, 17, 3, 2, 72, (12, 12, 12), True),
    (3, 5, 5, 5, 16, (4,), True), (1, 33, 7, 1, 24, (3, 4, 5), False), (2, 9, 4, 4, 40, (20,), True), (1, 77, 16, 16, 96, (13, 30), False),
    (5, 3, 2, 8, 64, (8, 8, 8, 8), True), (1, 4, 3, 3, 256, (128,), False), (2, 2, 9, 9, 200, (40, 20), True), (1, 2, 255, 300, 32, (9, 4), False),
    (1, 3, 2, 2, 136, (1, 1, 1, 1), False), (400, 16, 3, 3, 72, (36,), False), (1, 1, 1100, 0, 8, (4,), True),
]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("case", ROPES)
def test_norm_and_rotation(F, case, norm):
    batch, tokens, hq, hk, dim, pairs, halves = case
    q, k = rand(batch, hq, tokens, dim, seed=1), rand(batch, hk, tokens, dim, seed=2, scale=30.0) if hk else None
    g = [(1 + 0.3 * torch.randn(dim, device="cuda")) if norm else None for _ in range(2)]
    for shared in (1, batch):
        positions = torch.randint(-50, 5000, (shared, tokens, len(pairs)), device="cuda", dtype=torch.int32)
        check_rope(F, q, k, pairs, positions, g, norm=norm, halves=halves)


def test_norm_alone_and_missing_parts(F):
    q, k = rand(2, 3, 5, 72, seed=3), rand(2, 1, 5, 72, seed=4)
    check_rope(F, q, k, (), None)
    check_rope(F, q, None, (), None, (torch.rand(72, device="cuda"), None))
    check_rope(F, q, k, (2,), torch.zeros(1, 5, 1, device="cuda", dtype=torch.int32), (None, torch.rand(72, device="cuda")))
    out, _ = F.fb4_qk_norm_rope(q, None, None, None, (), norm=False)
    assert torch.equal(out, q)


@pytest.mark.parametrize("position", [2 ** 31 - 1, -2 ** 31, 1 << 20, 123456789])
def test_far_positions(F, position):
    q = rand(1, 2, 4, 64, seed=5)
    check_rope(F, q, q.clone(), (16, 16), torch.full((1, 4, 2), position, device="cuda", dtype=torch.int32))


def test_views(F):
    """Views of a packed projection, in the order that temporal attention takes, a batch of one sequence, rows far apart."""
    packed = rand(6, 11, 3 * 4, 48, seed=6)                       # [frames][tokens][q | k | v heads][dim]
    pos = torch.arange(11, device="cuda", dtype=torch.int32).view(1, 11, 1)
    x = packed.permute(0, 2, 1, 3)
    check_rope(F, x[:, :4], x[:, 4:8], (24,), pos)
    x = packed.permute(1, 2, 0, 3)                                # [tokens][heads][frames][dim]
    check_rope(F, x[:, :4], x[:, 4:8], (4, 20), torch.randint(0, 99, (11, 6, 2), device="cuda", dtype=torch.int32), halves=True)
    one = rand(1, 4, 11, 48, seed=7)
    check_rope(F, one.expand(5, 4, 11, 48), one[:, :1].expand(5, 3, 11, 48), (24,), pos)
    wide = rand(2, 3, 7, 4096, seed=8)
    check_rope(F, wide[..., 1024:1088], wide[..., 8:72], (32,), pos[:, :7])
    with pytest.raises(F.Fb4Error) as e:
        F.fb4_qk_norm_rope(wide[..., 4:68], None, pos[:, :7], torch.ones(32, device="cuda", dtype=torch.float64), (32,))
    assert e.value.code == F.ERR_UNSUPPORTED                       # rows that are not 16-byte aligned
    with pytest.raises(F.Fb4Error) as e:
        F.fb4_qk_norm_rope(rand(1, 2, 64, 8).transpose(2, 3), None, None, None, ())
    assert e.value.code == F.ERR_UNSUPPORTED                       # channels that are not contiguous


def test_values_stay_in_their_row(F):
    """Inf and NaN, squares beyond fp32, zero rows: each as the definition has it, its neighbours untouched."""
    q = rand(1, 6, 8, 72, seed=9)
    q[0, 0, 1, 5] = math.inf
    q[0, 1, 2, 71] = math.nan
    q[0, 2, 3] *= 2.0 ** 100
    q[0, 3, 4] *= 2.0 ** -120
    q[0, 4, 5] = 0
    q[0, 5, 6] = 3.0e38
    pos = torch.randint(0, 64, (1, 8, 2), device="cuda", dtype=torch.int32)
    for eps in (1e-6, 0.0):
        check_rope(F, q, q.flip(1).contiguous(), (10, 20), pos, eps=eps)
        check_rope(F, q, q.flip(1).contiguous(), (10, 10), pos, eps=eps, halves=True)
    # without the norm an Inf stays in its own pair, and channels that are not turned keep their values
    x = rand(1, 1, 2, 64, seed=10)
    x[0, 0, 0, 63] = math.inf
    x[0, 0, 1, 40] = math.nan
    out, _ = F.fb4_qk_norm_rope(x, None, torch.ones(1, 2, 1, device="cuda", dtype=torch.int32), torch.ones(8, device="cuda", dtype=torch.float64), (8,), norm=False)
    assert torch.equal(out[..., 16:].view(torch.int16), x[..., 16:].view(torch.int16)) and out[..., :16].isfinite().all()


# ------------------------------------------------------------------------------------------------ choice of blocks
def select_reference(q, k, top, block_q, block_k, lens):
    batch, heads, tq, dim = q.shape
    share, tk = heads // k.shape[1], k.shape[2]
    nq = -(-tq // block_q)
    blocks = torch.full((batch, heads, nq, top), -1, dtype=torch.int32)
    scores = torch.full((batch, heads, nq, top), math.nan)
    q, k = q.double().cpu(), k.double().cpu()
    for b in range(batch):
        lq, lk = (tq, tk) if lens is None else (min(max(int(lens[b, 0]), 0), tq), min(max(int(lens[b, 1]), 0), tk))
        for h in range(heads):
            km = [k[b, h // share, j:min(j + block_k, lk)].mean(0) for j in range(0, lk, block_k)]
            for i in range(0, lq, block_q):
                qm = q[b, h, i:min(i + block_q, lq)].mean(0)
                s = [float((qm * m).sum()) for m in km]
                best = sorted(range(len(s)), key=lambda j: (math.isnan(s[j]), -s[j] if not math.isnan(s[j]) else 0, j))[:top]
                for at, j in enumerate(sorted(best)):
                    blocks[b, h, i // block_q, at] = j
                    scores[b, h, i // block_q, at] = s[j]
    return blocks, scores


def check_select(F, q, k, top, block_q, block_k, lens=None):
    ref, ref_scores = select_reference(q, k, top, block_q, block_k, lens)
    guard = torch.full((ref.numel() + 64,), -9, dtype=torch.int32, device="cuda")
    blocks = guard[:ref.numel()].view(ref.shape)
    got, scores = F.fb4_select_key_blocks(q, k, top, block_q, block_k, lens, blocks=blocks, want_scores=True)
    alone = F.fb4_select_key_blocks(q, k, top, block_q, block_k, lens)
    torch.cuda.synchronize()
    assert got is blocks and (guard[ref.numel():] == -9).all()
    assert torch.equal(blocks.cpu(), ref) and torch.equal(alone, blocks)
    # 64-bit sums of at most 128 + 128 terms, then one rounding to fp32
    mass = ref_scores.double().abs() + 1e-12
    off = (scores.cpu().double() - ref_scores.double()).abs()
    assert ((off <= mass * 2.0 ** -23) | (ref_scores.isnan() & scores.cpu().isnan()) | (scores.cpu() == ref_scores)).all()


@pytest.mark.parametrize("case", [
    # batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, top
    (1, 1, 1, 1, 1, 8, 64, 64, 1), (1, 1, 1, 1, 700, 128, 128, 64, 3), (2, 4, 2, 200, 300, 64, 64, 128, 2), (1, 3, 1, 129, 65, 72, 128, 64, 5),
    (3, 2, 2, 64, 128, 16, 64, 64, 1), (1, 2, 2, 1350, 1350, 72, 64, 64, 6), (2, 6, 3, 127, 1025, 96, 64, 128, 9), (1, 1, 1, 300, 4100, 40, 128, 64, 64),
    (1, 2, 1, 2100, 129, 104, 64, 64, 3), (2, 1, 1, 65, 2000, 24, 64, 64, 32)])
def test_choice(F, case):
    b, h, hk, tq, tk, dim, bq, bk, top = case
    q, k = rand(b, h, tq, dim, seed=11), rand(b, hk, tk, dim, seed=12)
    check_select(F, q, k, top, bq, bk)
    lens = torch.tensor([[max(tq - 30 * i, 0), max(tk - 70 * i - 1, 0)] for i in range(b)], dtype=torch.int32, device="cuda")
    for x, which in ((q, 0), (k, 1)):
        for i in range(b):
            x[i, :, int(lens[i, which]):] = math.nan       # what lies behind is not read
    check_select(F, q, k, top, bq, bk, lens)


def test_choice_ties_nans_and_empty_sequences(F):
    k = torch.ones(2, 2, 1000, 32, device="cuda").bfloat16()
    q = torch.ones(2, 2, 200, 32, device="cuda").bfloat16()
    check_select(F, q, k, 5, 64, 64)                        # equal scores: the first
    q[:, 1] = -1
    k[0, 0, 128:192] = 2
    k[0, 0, 640:704] = 2
    k[1, 0, 3] = math.nan                                    # a block whose score is no number is last
    k[1, 1, 500] = math.inf
    check_select(F, q, k, 3, 64, 64)
    check_select(F, q, k, 16, 64, 64)
    check_select(F, q, k, 40, 64, 64)                        # more places than blocks
    q[0, 0, 70] = math.nan                                   # no number anywhere: the first
    check_select(F, q, k, 4, 64, 64)
    q[:] = 0
    q[0, 0, 0, 0] = -0.0
    check_select(F, q, torch.where(k == 1, -k, k).nan_to_num(1.0, 1.0), 4, 128, 128)   # +0 and -0 are one score
    for lens in ([[0, 1000], [200, 0]], [[-5, 5000], [3000, 1]]):
        check_select(F, rand(2, 2, 200, 32, seed=13), rand(2, 2, 1000, 32, seed=14), 4, 64, 64, torch.tensor(lens, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("blocks", [1, 63, 64, 65, 1000, 1024, 1025, 2048])
def test_choice_among_many_blocks(F, blocks):
    tokens = 64 * blocks - 5
    k = rand(1, 1, tokens, 16, seed=15)
    q = rand(1, 2, 130, 16, seed=16)
    for top in (1, max(1, blocks // 3), blocks):
        check_select(F, q, k, top, 64, 64)


# ------------------------------------------------------------------------------------------------ attention
def attention_reference(q, k, v, blocks, scale, block_q, block_k, lens):
    """(out [batch][heads][tokens][dim], bound, lse, bound, rows that are written) in 64 bits."""
    batch, heads, tq, dim = q.shape
    share, tk = heads // k.shape[1], k.shape[2]
    out, bound = torch.zeros(batch, heads, tq, dim, dtype=torch.float64, device="cuda"), torch.zeros(batch, heads, tq, dim, dtype=torch.float64, device="cuda")
    lse, lse_bound = torch.zeros(batch, heads, tq, dtype=torch.float64, device="cuda"), torch.zeros(batch, heads, tq, dtype=torch.float64, device="cuda")
    live = torch.zeros(batch, heads, tq, dtype=torch.bool, device="cuda")
    listed = None if blocks is None else blocks.tolist()
    for b in range(batch):
        lq, lk = (tq, tk) if lens is None else (min(max(int(lens[b, 0]), 0), tq), min(max(int(lens[b, 1]), 0), tk))
        live[b, :, :lq] = True
        for h in range(heads):
            for i0 in range(0, lq, block_q):
                i1 = min(i0 + block_q, lq)
                chosen = range(-(-lk // block_k)) if listed is None else listed[b][h][i0 // block_q]
                keys = [j for c in chosen if 0 <= c for j in range(c * block_k, min((c + 1) * block_k, lk))]
                if not keys:
                    lse[b, h, i0:i1] = -math.inf
                    continue
                at = torch.tensor(keys, device="cuda")
                qs, ks, vs = q[b, h, i0:i1].double(), k[b, h // share].index_select(0, at).double(), v[b, h // share].index_select(0, at).double()
                s = scale * (qs @ ks.T)
                # A weight: its score's dim products and sums in fp32, the power (argument and result), one rounding to bf16.
                # The sum of n positive weights: 16 of a group of 32 keys per lane, then one addition per group, each off by at most
                # 2^-24 of the sum: n / 32 + 16, and a few more where halves and parts meet.
                weight = (dim + 8) * 2.0 ** -23 * scale * (qs.abs() @ ks.abs().T).amax(-1, keepdim=True) + 2.0 ** -18 + (len(keys) / 32 + 64) * 2.0 ** -24
                total = torch.logsumexp(s, -1, keepdim=True)
                p = torch.exp(s - total)
                dead = total == -math.inf
                p = torch.where(dead, 0.0, p)
                out[b, h, i0:i1] = p @ vs
                bound[b, h, i0:i1] = (p @ vs.abs()) * (BF16 + 2 * weight) + BF16 * (p @ vs).abs() * (1 + BF16) + TINY
                lse[b, h, i0:i1], lse_bound[b, h, i0:i1] = total.squeeze(-1), (weight + 2.0 ** -21 * total.abs()).squeeze(-1)
    return out, bound, lse, lse_bound, live


def check_attention(F, q, k, v, blocks=None, scale=None, block_q=64, block_k=64, lens=None, out=None):
    batch, heads, tq, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    if out is None:
        flat = torch.full((batch * tq * heads * dim + 64,), -7.0, device="cuda", dtype=torch.bfloat16)
        out = flat[:-64].view(batch, tq, heads, dim)
    else:
        flat = None
        out.fill_(-7.0)
    lse = torch.full((batch * heads * tq + 64,), -7.0, device="cuda")
    got, got_lse = F.fb4_block_attention(q, k, v, blocks, scale, block_q, block_k, lens, out=out, lse=lse[:-64].view(batch, heads, tq))
    torch.cuda.synchronize()
    assert (lse[-64:] == -7.0).all() and (flat is None or (flat[-64:] == -7.0).all())
    ref, bound, ref_lse, lse_bound, live = attention_reference(q, k, v, blocks, scale, block_q, block_k, lens)
    got = got.permute(0, 2, 1, 3).double()
    what = (tuple(q.shape), tuple(k.shape), block_q, block_k)
    right = agree(got, ref, bound, live.unsqueeze(-1)), agree(got_lse.double(), ref_lse, lse_bound, live)
    kept = bool((got[~live] == -7.0).all()), bool((got_lse[~live] == -7.0).all())   # rows behind the last query
    assert right == (True, True) and kept == (True, True), what
    return out


def some_blocks(shape, blocks, seed=0):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.stack([torch.randperm(blocks, generator=g)[:shape[-1]].sort().values for _ in range(math.prod(shape[:-1]))]).view(shape).int().cuda()


@pytest.mark.parametrize("dim", list(range(8, 129, 8)))
def test_attention_channels(F, dim):
    q, k, v = rand(2, 2, 150, dim, seed=21), rand(2, 2, 333, dim, seed=22), rand(2, 2, 333, dim, seed=23)
    for bq, bk in ((64, 64), (128, 128)):
        check_attention(F, q, k, v, block_q=bq, block_k=bk)
        check_attention(F, q, k, v, some_blocks((2, 2, -(-150 // bq), 2), -(-333 // bk), dim), block_q=bq, block_k=bk)


@pytest.mark.parametrize("tq", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300])
@pytest.mark.parametrize("tk", [1, 15, 16, 63, 64, 65, 127, 128, 129, 200])
def test_attention_lengths(F, tq, tk):
    q, k, v = rand(1, 2, tq, 72, seed=24), rand(1, 1, tk, 72, seed=25), rand(1, 1, tk, 72, seed=26)
    for bq, bk in ((64, 128), (128, 64)):
        check_attention(F, q, k, v, block_q=bq, block_k=bk)


@pytest.mark.parametrize("tokens", [4000, 70000])
@pytest.mark.parametrize("case", [(1, 1, 1), (3, 4, 2), (2, 24, 8)])
def test_single_queries_over_long_sequences(F, tokens, case):
    b, h, hk = case
    q, k, v = rand(b, h, 1, 64, seed=27), rand(b, hk, tokens, 64, seed=28), rand(b, hk, tokens, 64, seed=29)
    check_attention(F, q, k, v)
    check_attention(F, q, k, v, some_blocks((b, h, 1, 37), -(-tokens // 64), 3))
    lens = torch.tensor([[1, tokens - 1000 * i - 17] for i in range(b)], dtype=torch.int32, device="cuda")
    check_attention(F, q, k, v, lens=lens, block_k=128)


def test_attention_lists(F):
    """Any order, entries without a key, one block twice, lists that name nothing."""
    q, k, v = rand(1, 1, 320, 64, seed=30), rand(1, 1, 500, 64, seed=31), rand(1, 1, 500, 64, seed=32)
    lists = torch.tensor([[7, 0, 3, 5], [-1, -1, -1, -1], [2, 2, 2, 2], [8, 1 << 30, -2 ** 31, 4], [7, 7, -1, 0]], dtype=torch.int32, device="cuda").view(1, 1, 5, 4)
    check_attention(F, q, k, v, lists)
    check_attention(F, q, k, v, lists, lens=torch.tensor([[300, 130]], dtype=torch.int32, device="cuda"))
    check_attention(F, q, k, v, torch.empty(1, 1, 5, 0, dtype=torch.int32, device="cuda"))
    check_attention(F, q, k[:, :, :0].contiguous(), v[:, :, :0])
    long = torch.randint(-1, 9, (1, 1, 5, 3000), device="cuda", dtype=torch.int32)      # longer than there are blocks
    check_attention(F, q, k, v, long)


def test_attention_padded_batches(F):
    """What lies behind a sequence's end has no part in it, whatever it holds, and rows behind the last query stay."""
    q, k, v = rand(4, 2, 200, 72, seed=33), rand(4, 2, 260, 72, seed=34), rand(4, 2, 260, 72, seed=35)
    lens = torch.tensor([[200, 260], [130, 65], [1, 1], [0, 0]], dtype=torch.int32, device="cuda")
    for i, (a, b) in enumerate(lens.tolist()):
        q[i, :, a:] = math.nan
        k[i, :, b:] = math.inf
        v[i, :, b:] = math.nan
    for bq, bk in ((64, 64), (128, 128)):
        check_attention(F, q, k, v, lens=lens, block_q=bq, block_k=bk)
    check_attention(F, q, k, v, some_blocks((4, 2, 4, 3), 5, 1), lens=lens)
    lens[3, 0] = 200
    lens[2, 1] = -4
    check_attention(F, q.nan_to_num(0.5), k, v, lens=lens)                    # queries without a key: zeros, -Inf


def test_attention_values_stay_where_they_belong(F):
    """A NaN or Inf in one head's blocks reaches the rows that attend it and no others; rows of a tile's padding do not."""
    q, k, v = rand(1, 3, 130, 40, seed=36), rand(1, 3, 300, 40, seed=37), rand(1, 3, 300, 40, seed=38)
    k[0, 1, 70, 39] = math.nan
    v[0, 2, 299, 0] = math.inf
    k[0, 2, 10, :] = 0
    q[0, 0, 5, 0] = math.nan
    lists = torch.tensor([[0, 1, 2], [0, 2, 4], [3, 4, -1]], dtype=torch.int32, device="cuda").view(1, 1, 3, 3).expand(1, 3, 3, 3).contiguous()
    check_attention(F, q, k, v, lists)
    big = q.clone()
    big[0, 0] *= 2.0 ** 60                                                     # one key takes all the weight
    check_attention(F, big.nan_to_num(1.0), k.nan_to_num(1.0), v.nan_to_num(1.0, 1.0))
    low = torch.full_like(k, -3.0e38)                                          # scores of the type's lowest value: -Inf in fp32
    out = F.fb4_block_attention(torch.full_like(q, 3.0e38), low, v.nan_to_num(1.0, 1.0), block_q=64, block_k=64)
    assert (out == 0).all()


@pytest.mark.parametrize("scale", [1e-6, 0.03, 1.0, 50.0])
def test_attention_scales_and_rising_scores(F, scale):
    """Scores that rise along the keys, by little and by much: the running maximum follows."""
    q, k, v = rand(1, 2, 96, 64, seed=39), rand(1, 2, 700, 64, seed=40), rand(1, 2, 700, 64, seed=41)
    k = (k.float() + q[:, :, :1].float() * torch.linspace(-1, 1, 700, device="cuda").view(1, 1, -1, 1)).bfloat16()
    check_attention(F, q, k, v, scale=scale)
    check_attention(F, q, k.flip(2).contiguous(), v, scale=scale, block_q=128, block_k=128)


def test_attention_strides(F):
    """Values out of a packed projection, outputs into part of a wider row, either order of heads and tokens."""
    q, k = rand(2, 4, 100, 64, seed=42), rand(2, 2, 190, 64, seed=43)
    packed = rand(2, 190, 5 * 2, 64, seed=44)
    v = packed[:, :, 4:6].permute(0, 2, 1, 3)
    dense = check_attention(F, q, k, v.contiguous())
    assert torch.equal(check_attention(F, q, k, v), dense)
    wide = torch.zeros(2, 100, 4, 200, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(check_attention(F, q, k, v, out=wide[..., 64:128]), dense)
    assert (wide[..., :64] == 0).all() and (wide[..., 128:] == 0).all()
    other = torch.zeros(2, 4, 100, 64, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(check_attention(F, q, k, v, out=other.permute(0, 2, 1, 3)), dense)
    check_attention(F, q, k, v[:, :1].expand(2, 2, 190, 64))                   # one value head for both
    for bad in (packed[:, :, 4:6, :60].permute(0, 2, 1, 3), packed.view(2, 190, 640)[:, :, 4:132].reshape(2, 190, 2, 64).permute(0, 2, 3, 1)):
        with pytest.raises(F.Fb4Error):
            F.fb4_block_attention(q, k, bad)


def test_offsets_beyond_32_bits(F):
    """Keys and values of more than 2^32 bytes in one head: the last blocks."""
    tokens = (1 << 24) + 5000
    k = torch.zeros(1, 1, tokens, 128, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros(1, 1, tokens, 128, device="cuda", dtype=torch.bfloat16)
    k[:, :, -6000:], v[:, :, -6000:] = rand(1, 1, 6000, 128, seed=45), rand(1, 1, 6000, 128, seed=46)
    q = rand(1, 1, 70, 128, seed=47)
    last = (tokens - 1) // 128
    lists = torch.tensor([last, last - 3, 0, 17, last - 40], dtype=torch.int32, device="cuda").view(1, 1, 1, 5)
    check_attention(F, q, k, v, lists, block_q=128, block_k=128)
    x = v[:, :, :tokens].view(1, 1, tokens, 128)
    out, _ = F.fb4_qk_norm_rope(x, None, None, None, (), norm=False)
    assert torch.equal(out[:, :, -6000:], x[:, :, -6000:])


def test_two_streams_and_graphs(F):
    """A captured chain, replayed with other inputs and eager work between, gives what the eager calls give, each time."""
    q, k, v = rand(1, 4, 700, 64, seed=50), rand(1, 4, 700, 64, seed=51), rand(1, 4, 700, 64, seed=52)
    one = rand(1, 4, 1, 64, seed=53)
    pos = torch.arange(700, device="cuda", dtype=torch.int32).view(1, 700, 1)
    freqs = 100.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)

    def chain():
        a, b = F.fb4_qk_norm_rope(q, k, pos, freqs, (32,))
        blocks = F.fb4_select_key_blocks(a, b, 3, 64, 64)
        return blocks, F.fb4_block_attention(a, b, v, blocks, block_q=64, block_k=64), F.fb4_block_attention(one, b, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            held = chain()
    torch.cuda.synchronize()
    for i in range(4):
        q.copy_(rand(1, 4, 700, 64, seed=60 + i))
        k.copy_(rand(1, 4, 700, 64, seed=70 + i))
        v.copy_(rand(1, 4, 700, 64, seed=80 + i))
        graph.replay()
        eager = chain()
        torch.cuda.synchronize()
        for a, b in zip(held, eager):
            assert torch.equal(a, b), i
    # on a stream that is not the current one, its workspace with it
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [F.fb4_block_attention(one, k, v, stream=s) for s in streams] + [F.fb4_block_attention(one, k, v)]
        lists = [F.fb4_select_key_blocks(q, k, 3, 64, 64, stream=s) for s in streams] + [F.fb4_select_key_blocks(q, k, 3, 64, 64)]
        torch.cuda.synchronize()
        assert all(torch.equal(g, got[-1]) for g in got) and all(torch.equal(x, lists[-1]) for x in lists)


@pytest.mark.parametrize("dim", [40, 64, 72, 104, 128])
def test_padding_leaves_no_trace(F, dim):
    """Rows behind a sequence's end change no bit of the others, not even by the rounding of what a wavefront shares."""
    lens = torch.tensor([[70, 200], [129, 65], [1, 333]], dtype=torch.int32, device="cuda")
    got = []
    for fill in (0.0, 3e30, math.inf, math.nan):
        q, k, v = rand(3, 2, 150, dim, seed=100), rand(3, 2, 333, dim, seed=101), rand(3, 2, 333, dim, seed=102)
        for i, (a, b) in enumerate(lens.tolist()):
            q[i, :, a:], k[i, :, b:], v[i, :, b:] = fill, fill, fill
        for bq, bk in ((64, 64), (128, 128)):
            blocks, scores = F.fb4_select_key_blocks(q, k, 2, bq, bk, lens, want_scores=True)
            got.append((blocks, scores.nan_to_num(-1.0), *F.fb4_block_attention(q, k, v, blocks, None, bq, bk, lens, want_lse=True),
                        F.fb4_block_attention(q, k, v, None, None, bq, bk, lens)))
    for i in range(2, len(got)):
        assert all(torch.equal(a, b) for a, b in zip(got[i], got[i % 2])), i


@pytest.mark.parametrize("block_q", [64, 128])
@pytest.mark.parametrize("dim", [40, 72, 104, 128])
def test_shared_lists(F, dim, block_q):
    """Lists long enough for several workgroups each: ragged sequences, entries without a key in some parts or all."""
    lens = torch.tensor([[200, 4000], [77, 2049], [1, 64], [200, 0]], dtype=torch.int32, device="cuda")
    q, k, v = rand(4, 2, 200, dim, seed=110), rand(4, 1, 4000, dim, seed=111), rand(4, 1, 4000, dim, seed=112)
    blocks = -(-200 // block_q)
    assert F.binding._lib.fb4_block_attention_workspace(4, 2, 1, 200, 4000, dim, F.binding.ALL_BLOCKS, block_q, 64) > 0
    check_attention(F, q, k, v, None, None, block_q, 64, lens)
    lists = some_blocks((4, 2, blocks, 40), 63, 7)
    lists[0, 0, 0, :25] = -1
    lists[0, 1, 0, 5:] = -1
    lists[1, 0] = -1
    assert F.binding._lib.fb4_block_attention_workspace(4, 2, 1, 200, 4000, dim, 40, block_q, 64) > 0
    check_attention(F, q, k, v, lists, None, block_q, 64, lens)


def test_parts_of_many_rows(F):
    """On both sides of the eight parts from which a row's join is a workgroup's."""
    for tokens, dim, more in ((2368, 8, True), (2368, 64, False)):
        q, k, v = rand(1, 2, tokens, dim, seed=120), rand(1, 2, 640, dim, seed=121), rand(1, 2, 640, dim, seed=122)
        g = torch.Generator()
        g.manual_seed(dim)
        lists = torch.randint(-1, 10, (1, 2, tokens // 64, 40), generator=g).int().cuda()
        size = F.binding._lib.fb4_block_attention_workspace(1, 2, 2, tokens, 640, dim, 40, 64, 64)
        assert size > 0 and (size > 8 * 2 * tokens * (dim + 2) * 4) == more
        check_attention(F, q, k, v, lists)


def test_given_workspaces(F):
    q, k, v = rand(1, 2, 1, 64, seed=130), rand(1, 2, 5000, 64, seed=131), rand(1, 2, 5000, 64, seed=132)
    lib = F.binding._lib
    size = lib.fb4_block_attention_workspace(1, 2, 2, 1, 5000, 64, F.binding.ALL_BLOCKS, 64, 64)
    held = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    got = F.fb4_block_attention(q, k, v, None, None, 64, 64, workspace=held[:size])
    assert torch.equal(got, F.fb4_block_attention(q, k, v, None, None, 64, 64)) and (held[size:] == 0xA5).all()
    with pytest.raises(F.Fb4Error):
        F.fb4_block_attention(q, k, v, None, None, 64, 64, workspace=held[:size - 1])
    with pytest.raises(F.Fb4Error):
        F.fb4_block_attention(q, k, v, None, None, 64, 64, workspace=held[8:])
    size = lib.fb4_select_key_blocks_workspace(1, 2, 2, 1, 5000, 64, 64, 64)
    held = torch.full((size + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    lists = F.fb4_select_key_blocks(q, k, 5, 64, 64, workspace=held[:size])
    assert torch.equal(lists, F.fb4_select_key_blocks(q, k, 5, 64, 64)) and (held[size:] == 0xA5).all()
    with pytest.raises(F.Fb4Error):
        F.fb4_select_key_blocks(q, k, 5, 64, 64, workspace=held[:size - 1])


def test_both_bindings_answer_alike(F):
    """The calls through the C module and through ctypes: the same results, the same refusals."""
    B = F.binding
    if B._heads_call is B.HeadsCall:
        pytest.skip("no C module")
    qkv = rand(2, 130, 6, 64, seed=140).permute(0, 2, 1, 3)
    q, k, v = qkv[:, :2].contiguous(), qkv[:, 2:4].contiguous(), qkv[:, 4:]
    lens = torch.tensor([[130, 100], [70, 130]], dtype=torch.int32, device="cuda")
    pos = torch.arange(130, device="cuda", dtype=torch.int32).view(1, 130, 1)
    freqs = 50.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)
    calls = [lambda: F.fb4_qk_norm_rope(qkv[:, :2], qkv[:, 2:4], pos, freqs, (32,)), lambda: F.fb4_qk_norm_rope(q, None, None, None, ()),
             lambda: F.fb4_qk_norm_rope(q, k, pos, freqs, (8, 24)), lambda: F.fb4_qk_norm_rope(q, k.float(), pos, freqs, (32,)),
             lambda: F.fb4_qk_norm_rope(q, k, pos.long(), freqs, (32,)), lambda: F.fb4_qk_norm_rope(q, k, pos, freqs[:31], (32,)),
             lambda: F.fb4_qk_norm_rope(q, k, pos, freqs, (32,), gamma_q=freqs.float()), lambda: F.fb4_qk_norm_rope(q, k, pos, freqs, (32,), pairing=2),
             lambda: F.fb4_qk_norm_rope(q.transpose(2, 3), None, None, None, ()), lambda: F.fb4_qk_norm_rope(q, k, pos, freqs, (32,), eps=-1.0)]
    for bq, bk in ((64, 64), (128, 64)):
        lists = F.fb4_select_key_blocks(q, k, 2, bq, bk, lens)
        calls += [lambda bq=bq, bk=bk: F.fb4_select_key_blocks(q, k, 2, bq, bk, lens, want_scores=True),
                  lambda bq=bq, bk=bk, x=lists: F.fb4_block_attention(q, k, v, x, None, bq, bk, lens, want_lse=True),
                  lambda bq=bq, bk=bk: F.fb4_block_attention(q, k, v, None, 0.3, bq, bk)]
    calls += [lambda: F.fb4_select_key_blocks(q, k, 2, 32, 64), lambda: F.fb4_select_key_blocks(qkv[:, :2], k, 2, 64, 64),
              lambda: F.fb4_select_key_blocks(q, k, 2, 64, 64, lens[:1]), lambda: F.fb4_select_key_blocks(q, k[:1], 2, 64, 64),
              lambda: F.fb4_select_key_blocks(q, k, 2, 64, 64, lens.long()), lambda: F.fb4_select_key_blocks(q, k, -1, 64, 64),
              lambda: F.fb4_block_attention(q, k, v[:, :, :129], None, 1.0, 64, 64), lambda: F.fb4_block_attention(q, k, v.transpose(2, 3), None, 1.0, 64, 64),
              lambda: F.fb4_block_attention(q, k, v, lists.long(), 1.0, 128, 64), lambda: F.fb4_block_attention(q, k, v, lists, 1.0, 64, 64),
              lambda: F.fb4_block_attention(q, k, v, None, 0.0, 64, 64), lambda: F.fb4_block_attention(q, k, v, None, math.nan, 64, 64),
              lambda: F.fb4_block_attention(q, k, v, None, 1.0, 64, 96), lambda: F.fb4_block_attention(q, k[:, :1], v, None, 1.0, 64, 64)]

    def answer(call):
        try:
            got = call()
        except F.Fb4Error as e:
            return str(e)
        return [x.nan_to_num(-1.0) if x.is_floating_point() else x for x in (got if isinstance(got, tuple) else (got,)) if x is not None]
    first = [answer(c) for c in calls]
    module = B._heads_call
    B._heads_call = B.HeadsCall
    try:
        second = [answer(c) for c in calls]
    finally:
        B._heads_call = module
    refused = 0
    for i, (a, b) in enumerate(zip(first, second)):
        refused += isinstance(a, str)
        assert a == b if isinstance(a, str) else all(torch.equal(x, y) for x, y in zip(a, b)), i
    assert refused == 8 + 6 + 8   # of the three calls, in the order above


def test_from_the_projection_to_the_quantizer(F):
    """As a layer uses them: norm and rotation out of the packed projection, salient tokens and key blocks from the same q and k,
    attention over the chosen blocks, its rows through the quantizer."""
    from fb4_inputs import DEFAULT_FORMATBOOK, synth
    from oracle import fb4_oracle as O
    frames, grid_h, grid_w, heads, dim = 4, 8, 16, 4, 64
    tokens = frames * grid_h * grid_w
    qkv = rand(1, tokens, 3 * heads, dim, seed=90)
    x = qkv.permute(0, 2, 1, 3)
    where = torch.stack(torch.meshgrid(*(torch.arange(n, device="cuda") for n in (frames, grid_h, grid_w)), indexing="ij"), -1).view(1, tokens, 3).int()
    pairs = (8, 12, 12)
    freqs = torch.cat([10000.0 ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n) for n in pairs])
    gamma = 1 + 0.1 * torch.randn(dim, device="cuda")
    q, k = F.fb4_qk_norm_rope(x[:, :heads], x[:, heads:2 * heads], where, freqs, pairs, gamma, gamma)
    for got, source in ((q, x[:, :heads]), (k, x[:, heads:2 * heads])):
        ref, mass = rope_reference(source, where, freqs, pairs, gamma, 1e-6, True, False)
        right = agree(got.double(), ref, (BF16 * ref.abs() + mass * 2.0 ** -16) * (1 + BF16) + TINY)
        assert right
    scores = F.fb4_attention_scores(q.view(heads, tokens, dim), k.view(heads, tokens, dim), 0)
    assert scores.isfinite().all()
    blocks = F.fb4_select_key_blocks(q, k, 3, 128, 64)
    assert torch.equal(blocks.cpu(), select_reference(q, k, 3, 128, 64, None)[0])
    out = check_attention(F, q, k, x[:, 2 * heads:], blocks, block_q=128, block_k=64)
    luts = F.fb4_build_luts(DEFAULT_FORMATBOOK)
    rows = out.view(tokens, heads * dim)
    codes, meta = F.fb4_quantize(luts, F.opts(), rows)
    torch.cuda.synchronize()
    codes_ref, meta_ref = O.quantize(DEFAULT_FORMATBOOK, synth.bf16_bits(rows))
    assert np.array_equal(codes.cpu().numpy(), codes_ref) and np.array_equal(meta.cpu().numpy().view(np.uint16), meta_ref)
    luts.free()


def test_outputs_of_another_stream_while_the_current_one_is_busy(F):
    """Outputs that the call makes itself, on a stream that waits for nothing: what the current one still has to do does not reach them."""
    q, k, v = rand(2, 4, 300, 64, seed=150), rand(2, 2, 500, 64, seed=151), rand(2, 2, 500, 64, seed=152)
    lens = torch.tensor([[300, 450], [77, 500]], dtype=torch.int32, device="cuda")
    pos = torch.arange(300, device="cuda", dtype=torch.int32).view(1, 300, 1)
    freqs = 50.0 ** (-torch.arange(32, device="cuda", dtype=torch.float64) / 32)
    calls = [lambda **a: F.fb4_block_attention(q, k, v, None, None, 64, 64, lens, want_lse=True, **a),
             lambda **a: F.fb4_block_attention(q, k, v, None, None, 128, 128, want_lse=True, **a),
             lambda **a: F.fb4_select_key_blocks(q, k, 3, 64, 64, lens, want_scores=True, **a),
             lambda **a: F.fb4_qk_norm_rope(q, q, pos, freqs, (32,), **a)]
    side, x = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for call in calls:
        ref = call()
        torch.cuda.synchronize()
        for _ in range(20):   # (some 30 ms)
            x @ x
        got = call(stream=side)
        side.synchronize()
        seen = [g.cpu() for g in got]      # behind the current stream's work, which is done with then
        torch.cuda.synchronize()
        for a, b, c in zip(got, ref, seen):
            a, b, c = (t.nan_to_num(-1.0) if t.is_floating_point() else t for t in (a, b, c))
            assert torch.equal(a, b) and torch.equal(a.cpu(), c)
    out = F.fb4_block_attention(q, k, v, None, None, 64, 64, lens, stream=side)
    side.synchronize()
    assert (out[1, 77:] == 0).all()


# Scores that are exact in fp32, of any size: what a weight is off by does not grow with them.
def exact_scores(first, second, key_first, key_second, v, scale):
    """Query i's score of key j is first * key_first[j] + second[i] * key_second[j].  (the scores; the call's first arguments)"""
    q, k = torch.zeros(1, 1, len(second), 64, dtype=torch.float64), torch.zeros(1, 1, len(key_first), 64, dtype=torch.float64)
    q[0, 0, :, 0], q[0, 0, :, 1] = first, torch.as_tensor(second, dtype=torch.float64)
    k[0, 0, :, 0], k[0, 0, :, 1] = torch.as_tensor(key_first, dtype=torch.float64), torch.as_tensor(key_second, dtype=torch.float64)
    s = q[0, 0] @ k[0, 0].T
    assert all(torch.equal(x, x.bfloat16().double()) for x in (q, k)) and torch.equal(s, s.float().double()) and scale == float(np.float32(scale))
    return s, q.bfloat16().cuda(), k.bfloat16().cuda(), v, scale


def check_exact_scores(F, s, q, k, v, scale, block_q=64, parts=False):
    """parts: the list is shared by several workgroups (not where there are as many as 1024 heads)."""
    if not parts:
        q = q.expand(1, 1024, -1, -1).contiguous()
    size = F.binding._lib.fb4_block_attention_workspace(1, q.shape[1], 1, q.shape[2], k.shape[2], 64, F.binding.ALL_BLOCKS, block_q, 64)
    assert (size > 0) == parts
    out, lse = F.fb4_block_attention(q, k, v, None, scale, block_q, 64, want_lse=True)
    assert agree(out, out[:, :, :1], 0) and agree(lse, lse[:, :1], 0)
    s, v64 = s.cuda() * scale, v[0, 0].double()
    total = torch.logsumexp(s, -1, keepdim=True)
    p = torch.softmax(s, -1)
    # A weight: the power's argument, of which 2^-22 is lost (above 2^-40 of the largest it is below 40), and its result; one
    # rounding to bf16.  The sum as in attention_reference.
    weight = 40 * 2.0 ** -22 + 2.0 ** -18 + (s.shape[1] / 32 + 64) * 2.0 ** -24
    bound = (p @ v64.abs()) * (BF16 + 2 * weight) + BF16 * (p @ v64).abs() * (1 + BF16) + TINY + 2.0 ** -40 * v64.abs().sum(0)
    right = agree(out[0, :, 0].double(), p @ v64, bound), agree(lse[0, 0].double(), total[:, 0], weight + 2.0 ** -21 * total[:, 0].abs())
    assert right == (True, True), ((out[0, :, 0].double() - p @ v64).abs() / bound).max()


def old_and_new_values(keys, new, seed):
    v = rand(1, 1, keys, 64, seed=seed)
    v[0, 0, :, 0], v[0, 0, new, 0] = 1, -1
    return v


LARGE_SCORES = [(2048, 2832, 0.125), (-2048, 2832, 0.125), (2048, 2048, 0.17), (1024, 1416, 0.125), (64, 96, 0.125)]   # log2 of a weight up to 2^20
LARGER_SCORES = [(2048, 6144, 0.125), (2048, 6112, 0.125), (-2048, 6112, 0.125), (2048, 8160, 0.5)]                   # beyond


@pytest.mark.parametrize("block_q", [64, 128])
@pytest.mark.parametrize("first,key,scale", LARGE_SCORES + LARGER_SCORES)
def test_large_scores_with_a_moving_maximum(F, first, key, scale, block_q):
    """Some of a row's weights are taken before its maximum moves and some after: both count relative to one reference."""
    scale = float(np.float32(scale))
    least = int(8 / (scale * 1.4427)) + 1
    second = list(range(least, least + 36))                      # what the late keys' scores have more
    for keys in (65, 300, 449):
        for late in ([keys - 1], [70 % keys, keys - 1], list(range(33, 64))):
            more = torch.zeros(keys)
            more[late] = 1
            check_exact_scores(F, *exact_scores(first, second, [key] * keys, more, old_and_new_values(keys, late, keys), scale), block_q)


@pytest.mark.parametrize("keys", [300, 2000])
def test_scores_on_both_sides_of_two_to_the_twentieth(F, keys):
    """A row's weights are formed one way up to 2^20 and another beyond: a row that begins below and ends above."""
    for sign in (1, -1):
        for below in (4.0, 20.0):
            scale = float(np.float32((2.0 ** 20 - sign * below) / (2.0 ** 22 * math.log2(math.e))))   # 0.1733: 1/4 per unit of a score
            more = torch.zeros(keys)
            more[keys // 2:] = 1
            more[-1] = 2
            v = old_and_new_values(keys, list(range(keys // 2, keys)), 9)
            second = [4, 8, 20, 30, 33, 36, 40, 44, 50, 60]
            check_exact_scores(F, *exact_scores(2048 * sign, second, [2048] * keys, more, v, scale), parts=keys > 300)


@pytest.mark.parametrize("first,key,scale", LARGE_SCORES + LARGER_SCORES)
def test_large_scores_in_parts(F, first, key, scale):
    """Parts of a list with maxima of their own: joined relative to one."""
    scale = float(np.float32(scale))
    second, keys = list(range(1, 40)), 2000
    for late in ([keys - 1], [100], list(range(640, 700)) + [1500]):
        more = torch.zeros(keys)
        more[late] = 1
        check_exact_scores(F, *exact_scores(first, second, [key] * keys, more, old_and_new_values(keys, late, 7), scale), parts=True)


def test_far_scores_that_are_neighbours(F):
    """Scores so far out that a step of theirs is more than a weight's range, whose products with the scale round to one number: the
    larger one takes all the weight."""
    rng, found = np.random.default_rng(5), 0
    low, high = 255 * 2.0 ** 16, 2.0 ** 16                           # scores about 2^33, 512 apart
    for scale in np.linspace(0.25, 0.27, 400).astype(np.float32) / np.float32(math.log2(math.e)):
        factor = np.float32(scale * np.float32(math.log2(math.e)))
        for j in rng.integers(0, 200, 4):
            a, b = np.float32(255 * 2.0 ** 25 + 512 * int(j)), np.float32(255 * 2.0 ** 25 + 512 * int(j + 1))
            if float(b) * float(factor) - float(a * factor) > 8 or found >= 12:
                continue
            found += 1
            more = torch.full((200,), float(j))
            more[150:] = float(j + 1)
            v = old_and_new_values(200, list(range(150, 200)), 11)
            check_exact_scores(F, *exact_scores(2.0 ** 16, [512.0] * 5, [255 * 2.0 ** 9] * 200, more, v, float(scale)))
    assert found == 12


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("keys", [200, 3000])
def test_scores_at_the_end_of_fp32(F, keys, sign):
    """Finite scores whose products with log2 e are not."""
    for order in (1, -1):
        k = torch.full((keys,), 1.5 * 2.0 ** 64)
        k[keys // 2:] = 1.75 * 2.0 ** 64
        if order < 0:
            k = k.flip(0)
        v = old_and_new_values(keys, list(range(keys // 2, keys)), 12)
        check_exact_scores(F, *exact_scores(sign * 2.0 ** 63, [1.0] * 3, k, [0.0] * keys, v, 1.0), parts=keys > 200)


@pytest.mark.parametrize("keys", [1, 40, 300, 3000])
def test_infinite_scores(F, keys):
    """A key whose score is +Inf: no number for the row's output, +Inf for its lse; a NaN beside it is a NaN; other rows as ever."""
    q, k, v = rand(1, 1, 40, 64, seed=160), rand(1, 1, keys, 64, seed=161), rand(1, 1, keys, 64, seed=162)
    q[..., 0], k[..., 0] = 0, 0
    ref, ref_lse = F.fb4_block_attention(q, k, v, None, None, 64, 64, want_lse=True)
    for at in {0, keys // 2, keys - 1}:
        far = k.clone()
        far[0, 0, at, 0] = 3e38
        row = q.clone()
        row[0, 0, 7, 0], row[0, 0, 33, 0], row[0, 0, 34, 0] = 3e38, -3e38, 3e38
        row[0, 0, 34, 5] = math.nan
        out, lse = F.fb4_block_attention(row, far, v, None, None, 64, 64, want_lse=True)
        others = torch.ones(40, dtype=torch.bool, device="cuda")
        others[[7, 33, 34]] = False
        assert out[0, 7].isnan().all() and lse[0, 0, 7] == math.inf
        assert out[0, 34].isnan().all() and lse[0, 0, 34].isnan()
        assert not out[0, 33].isnan().any() and ((lse[0, 0, 33] == -math.inf) == (keys == 1)) and not lse[0, 0, 33].isnan()
        assert agree(out[0, others].double(), ref[0, others].double(), 2 * BF16 * (ref[0, others].double().abs() + 1.0))
        assert agree(lse[0, 0, others].double(), ref_lse[0, 0, others].double(), 2.0 ** -18 + 2.0 ** -20 * ref_lse[0, 0, others].double().abs())


def test_numbers_that_c_would_cut_off(F):
    """By either way into the library: 2^32 + 64 is not 64, 2^64 + 2 not 2."""
    B = F.binding
    q, k, v = rand(1, 2, 100, 64, seed=170), rand(1, 2, 200, 64, seed=171), rand(1, 2, 200, 64, seed=172)
    pos, freqs = torch.zeros(1, 100, 1, device="cuda", dtype=torch.int32), torch.ones(8, device="cuda", dtype=torch.float64)
    lists, far = torch.zeros(1, 2, 1, 2, device="cuda", dtype=torch.int32), 2 ** 32
    calls = [lambda: F.fb4_select_key_blocks(q, k, 2, far + 64, 64), lambda: F.fb4_select_key_blocks(q, k, 2, 64, far + 64),
             lambda: F.fb4_select_key_blocks(q, k, 2, far + 64, 64, blocks=lists), lambda: F.fb4_select_key_blocks(q, k, 2 ** 64 + 2, 128, 64, blocks=lists),
             lambda: F.fb4_block_attention(q, k, v, lists, None, far + 128, 64), lambda: F.fb4_block_attention(q, k, v, None, None, 64, far + 64),
             lambda: F.fb4_qk_norm_rope(q, q, pos, freqs, (far + 8,)), lambda: F.fb4_qk_norm_rope(q, q, pos, freqs, (8,), pairing=far),
             lambda: F.fb4_qk_norm_rope(q, q, pos, freqs, (8,), pairing=2 ** 64 + 1)]
    module = B._heads_call
    try:
        for B._heads_call in {module, B.HeadsCall}:
            for i, call in enumerate(calls):
                with pytest.raises(F.Fb4Error):
                    call()
                    raise AssertionError(i)
    finally:
        B._heads_call = module


def test_rotation_in_place(F):
    """Row upon row an output may be its input; on memory that is read elsewhere it is refused."""
    pos = torch.randint(0, 99, (1, 333, 1), device="cuda", dtype=torch.int32)
    freqs = 50.0 ** (-torch.arange(36, device="cuda", dtype=torch.float64) / 36)
    for halves in (F.ROPE_ADJACENT, F.ROPE_HALVES):
        q, k = rand(3, 20, 333, 72, seed=180), rand(3, 11, 333, 72, seed=181)
        ref = F.fb4_qk_norm_rope(q, k, pos, freqs, (36,), pairing=halves)
        qi, ki = q.clone(), k.clone()
        got = F.fb4_qk_norm_rope(qi, ki, pos, freqs, (36,), pairing=halves, q_out=qi, k_out=ki)
        assert got[0] is qi and got[1] is ki and all(torch.equal(a, b) for a, b in zip(got, ref))
    packed = rand(2, 333, 3, 72, seed=182)
    view = packed.permute(0, 2, 1, 3)
    memory = packed.view(-1)
    for out in (memory[:2 * 333 * 72].view(2, 1, 333, 72), memory[-2 * 333 * 72:].view(2, 1, 333, 72)):
        for args in ((view[:, :1], None), (q[:2, :1].contiguous(), view[:, 1:2])):
            with pytest.raises(F.Fb4Error) as e:
                F.fb4_qk_norm_rope(*args, pos, freqs, (36,), q_out=out)
            assert e.value.code == F.ERR_INVALID_ARG
    with pytest.raises(F.Fb4Error):
        F.fb4_qk_norm_rope(q, q, pos, freqs, (36,), q_out=qi, k_out=qi)


def test_captured_on_a_stream_beside_the_captured_one(F):
    """A call on a second stream of a capture, with outputs of its own making: replays give what eager calls do."""
    q, k, v = rand(2, 4, 300, 64, seed=190), rand(2, 2, 500, 64, seed=191), rand(2, 2, 500, 64, seed=192)
    lens = torch.tensor([[300, 450], [77, 500]], dtype=torch.int32, device="cuda")
    main, side = torch.cuda.Stream(), torch.cuda.Stream()

    def both():
        side.wait_stream(torch.cuda.current_stream())
        lists = F.fb4_select_key_blocks(q, k, 3, 64, 64, lens, stream=side)
        a = F.fb4_block_attention(q, k, v, lists, None, 64, 64, lens, want_lse=True, stream=side)
        b = F.fb4_block_attention(q, k, v, None, None, 64, 64, lens, want_lse=True)
        del lists
        torch.cuda.current_stream().wait_stream(side)
        return (*a, *b)
    main.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(main):
        both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        held = both()
    for i in range(4):
        q.copy_(rand(2, 4, 300, 64, seed=200 + i))
        k.copy_(rand(2, 2, 500, 64, seed=210 + i))
        graph.replay()
        eager = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager)), i
