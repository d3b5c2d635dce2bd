"""The attention path between a video DiT's packed projection and its output projection, as timed and compared passes.

A layer's queries and keys are normalised per head and rotated by their positions in time, height and width
(`norm_rope`); block means of both choose, for every block of queries, the key blocks worth attending (`select`); the
attention runs over those blocks (`attention`) and writes the rows that the quantizer of the output projection reads.
Sizes: this repository's configurations (16 frames of 32 x 32 tokens with 24 heads of 128 channels, 17 frames of 30 x 45
tokens with 16 heads of 72 channels, 65536 tokens) and the range from one token up.

`own` false: the plain forms, in elementary torch operations; true: this package's entry points.
"""

import math

import torch

own = False

# A drawn case costs no more than the largest listed ones: elements of q and k, gathered key elements.
_CAP_ROWS = 65536 * (24 + 24) * 128
_CAP_GATHER = 24 * 512 * 16 * 128 * 128


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a few text tokens of a short prompt beside a clip: a call of almost only latency
        _rope("rope_text", 2, 77, 16, 16, 72, (36,), halves=True, packed=True, far=77),
        # the benchmark clip's spatial attention: per-frame queries and keys out of the packed projection, three axes
        _rope("rope_clip", 16, 1024, 24, 24, 128, (8, 28, 28), packed=True, far=64),
        # temporal attention of the 72-channel model: every position's frames, a permuted view of the packed projection
        _rope("rope_temporal", 1350, 17, 16, 16, 72, (12, 12, 12), halves=True, packed=True, temporal=True, far=45),
        # 65536 tokens in one sequence at far positions, part of the channels rotated, keys with fewer heads
        _rope("rope_long", 1, 65536, 24, 8, 128, (48,), far=1 << 20),
        # one frame's tokens, blocks of 64
        _select("select_frame", 2, 16, 1350, 1350, 72, 64, 64, 6, ragged=True),
        # the clip as one sequence (3D attention)
        _select("select_clip", 1, 24, 16384, 16384, 128, 128, 128, 16),
        # 65536 tokens, 1024 blocks of 64
        _select("select_long", 1, 24, 65536, 65536, 128, 64, 64, 64),
        # cross attention of a frame's tokens to a short text, every block, ragged text lengths
        _attention("attention_text", 4, 16, 16, 400, 120, 72, 64, 64, 0, ragged=True),
        # one query token (an appended token, a class token) over a long sequence's chosen blocks, shared key heads
        _attention("attention_single", 2, 24, 8, 1, 65536, 128, 64, 64, 128),
        # every frame of the 72-channel model by itself: 1350 tokens, a third of the blocks, padded frames
        _attention("attention_spatial", 17, 16, 16, 1350, 1350, 72, 64, 64, 7, ragged=True),
        # the clip as one sequence: an eighth of its key blocks
        _attention("attention_clip", 1, 24, 24, 16384, 16384, 128, 128, 128, 16),
        # 65536 tokens, a thirty-second of the key blocks
        _attention("attention_long", 1, 24, 24, 65536, 65536, 128, 128, 128, 16),
    ]


def _rope(name, batch, tokens, heads_q, heads_k, dim, axis_pairs, halves=False, packed=False, temporal=False, far=64):
    """packed: views of one [..., q | k | v] projection; temporal: batch and tokens exchanged in memory; far: positions."""
    return dict(kind="rope", name=name, batch=batch, tokens=tokens, heads_q=heads_q, heads_k=heads_k, dim=dim,
                axis_pairs=" ".join(str(p) for p in axis_pairs), halves=halves, packed=packed, temporal=temporal, far=far)


def _select(name, batch, heads, tokens_q, tokens_k, dim, block_q, block_k, top, ragged=False):
    return dict(kind="select", name=name, batch=batch, heads=heads, tokens_q=tokens_q, tokens_k=tokens_k, dim=dim,
                block_q=block_q, block_k=block_k, top=top, ragged=ragged)


def _attention(name, batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, top, ragged=False):
    """top: listed blocks per block of queries (0: no list, every block)."""
    return dict(kind="attention", name=name, batch=batch, heads=heads, heads_k=heads_k, tokens_q=tokens_q, tokens_k=tokens_k,
                dim=dim, block_q=block_q, block_k=block_k, top=top, ragged=ragged)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rope", "select", "attention", "attention", "attention"])
    dim = rng.choice([128, 128, 72, 64, 96, 8 * rng.randint(2, 16)])
    while True:
        heads = rng.choice([24, 16, rng.randint(1, 24)])
        if kind == "rope":
            batch, tokens, heads_k = _log_int(rng, 1, 1500), _log_int(rng, 1, 65536), rng.choice([heads, rng.randint(1, heads)])
            if batch * tokens * (heads + heads_k) * dim > _CAP_ROWS:
                continue
            halves, axes = rng.random() < 0.5, rng.choice([1, 2, 3])
            most = dim // 2
            pairs = most if rng.random() < 0.7 else rng.randint(axes, most)
            if halves:
                pairs = max(pairs // 4 * 4, 4)
            cut = sorted(rng.sample(range(1, pairs), axes - 1)) if axes > 1 else []
            split = [b - a for a, b in zip([0] + cut, cut + [pairs])]
            c = _rope("", batch, tokens, heads, heads_k, dim, split, halves, packed=rng.random() < 0.6, far=_log_int(rng, 16, 1 << 20))
            c["temporal"] = rng.random() < 0.3
        else:
            batch, tokens_k = _log_int(rng, 1, 32), _log_int(rng, 1, 65536)
            tokens_q = rng.choice([tokens_k, tokens_k, 1, _log_int(rng, 1, 65536)])
            block_q, block_k = rng.choice([64, 128]), rng.choice([64, 128])
            nq, nk = -(-tokens_q // block_q), -(-tokens_k // block_k)
            if batch * heads * (tokens_q + tokens_k) * dim > _CAP_ROWS:
                continue
            top = max(1, min(nk, _log_int(rng, 1, 128)))
            ragged = rng.random() < 0.4
            if kind == "select":
                c = _select("", batch, heads, tokens_q, tokens_k, dim, block_q, block_k, top, ragged)
            else:
                top = 0 if nk <= 16 and rng.random() < 0.5 else top
                heads_k = rng.choice([h for h in range(1, heads + 1) if heads % h == 0] + [heads] * 3)
                if batch * heads * nq * (top or nk) * block_k * max(dim, block_q) > _CAP_GATHER:
                    continue
                c = _attention("", batch, heads, heads_k, tokens_q, tokens_k, dim, block_q, block_k, top, ragged)
        del c["name"]
        return c


def _lens(case):
    """(queries, keys) of every sequence of a padded batch, the first at full length."""
    cut = lambda n, b: n - (b * 7919) % (n // 4 + 1)
    return [(cut(case["tokens_q"], b), cut(case["tokens_k"], b)) for b in range(case["batch"])]


def work(case):
    if case["kind"] == "rope":
        rows = case["batch"] * case["tokens"] * (case["heads_q"] + case["heads_k"])
        n = rows * case["dim"]
        return {"bytes": 4 * n + 4 * case["tokens"] * len(case["axis_pairs"].split()), "flops": 8 * n}
    lens = _lens(case) if case["ragged"] else [(case["tokens_q"], case["tokens_k"])] * case["batch"]
    nq = -(-case["tokens_q"] // case["block_q"])
    if case["kind"] == "select":
        n = sum(a + b for a, b in lens) * case["heads"] * case["dim"]
        scores = sum(-(-a // case["block_q"]) * -(-b // case["block_k"]) for a, b in lens) * case["heads"]
        return {"bytes": 2 * n + 4 * case["batch"] * case["heads"] * nq * case["top"], "flops": n + 2 * scores * case["dim"]}
    bytes_, flops = 0, 0
    for a, b in lens:
        keys = b if case["top"] == 0 else min(b, case["top"] * case["block_k"])
        touched = min(b * case["heads_k"], -(-a // case["block_q"]) * keys * case["heads"])
        bytes_ += 2 * case["dim"] * (2 * a * case["heads"] + 2 * touched)
        flops += 4 * a * keys * case["dim"] * case["heads"]
    return {"bytes": bytes_, "flops": flops}


# ------------------------------------------------------------------------------------------------ inputs
def _rows(g, batch, heads, tokens, dim, spread=1.0):
    """bf16 [batch][heads][tokens][dim]: noise on top of what neighbouring tokens share."""
    x = torch.randn(batch, heads, tokens, dim, device="cuda", generator=g, dtype=torch.bfloat16)
    runs = -(-tokens // 48)
    shared = torch.randn(batch, heads, runs, dim, device="cuda", generator=g, dtype=torch.bfloat16)
    return (x + 0.7 * shared.repeat_interleave(48, 2)[:, :, :tokens]).mul_(spread)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "rope":
        b, t, hq, hk, d = (case[n] for n in ("batch", "tokens", "heads_q", "heads_k", "dim"))
        first, second = (t, b) if case["temporal"] else (b, t)
        heads = hq + 2 * hk if case["packed"] else hq + hk
        x = torch.randn(first, second, heads, d, device="cuda", generator=g, dtype=torch.bfloat16)
        x *= torch.exp(0.5 * torch.randn(heads, d, device="cuda", generator=g)).bfloat16()   # channels of unlike size
        if case["packed"]:
            x = x.permute(1, 2, 0, 3) if case["temporal"] else x.permute(0, 2, 1, 3)
            s["q"], s["k"] = x[:, :hq], x[:, hq:hq + hk]
        else:
            x = x.permute(1, 2, 0, 3) if case["temporal"] else x.permute(0, 2, 1, 3)
            s["q"], s["k"] = x[:, :hq].contiguous(), x[:, hq:].contiguous()
        pairs = [int(p) for p in case["axis_pairs"].split()]
        s["axis_pairs"] = pairs
        s["freqs"] = torch.cat([10000.0 ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n) for n in pairs])
        s["positions"] = torch.randint(0, case["far"], (b if case["temporal"] else 1, t, len(pairs)), device="cuda", generator=g, dtype=torch.int32)
        s["gamma_q"] = 1 + 0.2 * torch.randn(d, device="cuda", generator=g)
        s["gamma_k"] = 1 + 0.2 * torch.randn(d, device="cuda", generator=g)
        s["q_out"], s["k_out"] = (torch.empty(b, h, t, d, device="cuda", dtype=torch.bfloat16) for h in (hq, hk))
        return s
    b, h, d, tq, tk = (case[n] for n in ("batch", "heads", "dim", "tokens_q", "tokens_k"))
    hk = case.get("heads_k", h)
    nq, nk = -(-tq // case["block_q"]), -(-tk // case["block_k"])
    s["q"], s["k"] = _rows(g, b, h, tq, d), _rows(g, b, hk, tk, d)
    lens = _lens(case) if case["ragged"] else [(tq, tk)] * b
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda") if case["ragged"] else None
    if case["kind"] == "select":
        s["blocks"] = torch.empty(b, h, nq, case["top"], dtype=torch.int32, device="cuda")
        s["scores"] = torch.empty(b, h, nq, case["top"], device="cuda")
        return s
    # values: the last part of a packed [tokens][k | v] projection, rows of [batch][tokens][2 * heads][dim]
    s["v"] = torch.randn(b, tk, 2 * hk, d, device="cuda", generator=g, dtype=torch.bfloat16)[:, :, hk:].permute(0, 2, 1, 3)
    s["blocks"] = None
    if case["top"]:
        # distinct blocks per block of queries, ascending, of the sequence's own; -1 where it has fewer
        have = torch.tensor([-(-k // case["block_k"]) for _, k in lens], device="cuda").view(b, 1, 1, 1)
        at = torch.arange(nk, device="cuda")
        order = torch.rand(b, h, nq, nk, device="cuda", generator=g).add_((at >= have).float()).argsort(-1)[..., :case["top"]]
        order = torch.where(order < have, order, nk).sort(-1).values
        s["blocks"] = torch.where(order < nk, order, -1).to(torch.int32)
    s["scale"] = d ** -0.5
    s["out"] = torch.zeros(b, tq, h, d, device="cuda", dtype=torch.bfloat16)
    s["lse"] = torch.zeros(b, h, tq, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _run_own(s)
    if s["kind"] == "rope":
        axis = torch.repeat_interleave(torch.arange(len(s["axis_pairs"]), device="cuda"), torch.tensor(s["axis_pairs"], device="cuda"),
                                       output_size=sum(s["axis_pairs"]))
        angle = s["positions"][..., axis].double() * s["freqs"]                  # [1 or batch][tokens][pairs]
        cos, sin = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
        return {"q": _rope_plain(s["q"], s["gamma_q"], cos, sin, s["halves"]), "k": _rope_plain(s["k"], s["gamma_k"], cos, sin, s["halves"])}
    return _select_plain(s) if s["kind"] == "select" else _attention_plain(s)


def _run_own(s):
    import paper_2603_02883_amd as F
    if s["kind"] == "rope":
        q, k = F.fb4_qk_norm_rope(s["q"], s["k"], s["positions"], s["freqs"], s["axis_pairs"], gamma_q=s["gamma_q"],
                                  gamma_k=s["gamma_k"], eps=1e-6, pairing=F.ROPE_HALVES if s["halves"] else F.ROPE_ADJACENT,
                                  q_out=s["q_out"], k_out=s["k_out"])
        return {"q": q, "k": k}
    if s["kind"] == "select":
        blocks, scores = F.fb4_select_key_blocks(s["q"], s["k"], s["top"], block_q=s["block_q"], block_k=s["block_k"], lens=s["lens"],
                                                 blocks=s["blocks"], scores=s["scores"])
        return {"blocks": blocks, "scores": scores}
    out, lse = F.fb4_block_attention(s["q"], s["k"], s["v"], blocks=s["blocks"], scale=s["scale"], block_q=s["block_q"],
                                     block_k=s["block_k"], lens=s["lens"], out=s["out"], lse=s["lse"])
    return {"out": out, "lse": lse}


def _rope_plain(x, gamma, cos, sin, halves):
    x = x.float()
    y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gamma
    p = cos.shape[-1]
    u, v = (y[..., :p], y[..., p:2 * p]) if halves else (y[..., 0:2 * p:2], y[..., 1:2 * p:2])
    a, b = u * cos - v * sin, u * sin + v * cos
    turned = torch.cat([a, b], -1) if halves else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, y[..., 2 * p:]], -1).bfloat16().contiguous()


def _means(x, block, lens):
    """Mean over the first lens[b] rows of every block of rows, in 64 bits: [batch][heads][blocks][dim]."""
    b, h, t, d = x.shape
    n = -(-t // block)
    x = torch.nn.functional.pad(x.double(), (0, 0, 0, n * block - t))
    inside = (torch.arange(n * block, device="cuda") < lens.view(b, 1, 1)).view(b, 1, n, block, 1)
    return torch.where(inside, x.view(b, h, n, block, d), 0.0).sum(3) / inside.sum(3).clamp(min=1)


def _lens_of(s):
    b = s["q"].shape[0]
    if s["lens"] is not None:
        return s["lens"][:, 0].long(), s["lens"][:, 1].long()
    return (torch.full((b,), s[n].shape[2], device="cuda") for n in ("q", "k"))


def _select_plain(s):
    b, h, tq, d = s["q"].shape
    q_lens, k_lens = _lens_of(s)
    score = _means(s["q"], s["block_q"], q_lens) @ _means(s["k"], s["block_k"], k_lens).transpose(2, 3).contiguous()
    n = score.shape[-1]
    have = ((k_lens + s["block_k"] - 1) // s["block_k"]).view(b, 1, 1, 1)
    score = score.masked_fill(torch.arange(n, device="cuda") >= have, -math.inf)
    order = score.sort(dim=-1, descending=True, stable=True).indices[..., :s["top"]]
    live = (torch.arange(score.shape[2], device="cuda") * s["block_q"] < q_lens.view(b, 1, 1)).unsqueeze(-1)
    order = torch.where((order < have) & live, order, n).sort(-1).values
    listed_score = score.gather(-1, order.clamp(max=n - 1)).masked_fill(order == n, math.nan)
    return {"blocks": torch.where(order < n, order, -1).to(torch.int32), "scores": listed_score.float()}


def _attention_plain(s):
    q, k, v, block_q, block_k = s["q"], s["k"], s["v"], s["block_q"], s["block_k"]
    (b, h, tq, d), (_, hk, tk, _) = q.shape, k.shape
    nq, nk = -(-tq // block_q), -(-tk // block_k)
    q_lens, k_lens = _lens_of(s)
    blocks = s["blocks"] if s["blocks"] is not None else torch.arange(nk, device="cuda").expand(b, h, nq, nk)
    at = blocks.clamp(0, nk - 1).long()
    batch, head = torch.arange(b, device="cuda").view(b, 1, 1, 1), (torch.arange(h, device="cuda") // (h // hk)).view(1, h, 1, 1)
    pad = (0, 0, 0, nk * block_k - tk)
    gathered = [torch.nn.functional.pad(x, pad).reshape(b, hk, nk, block_k, d)[batch, head, at].float().view(b * h * nq, -1, d) for x in (k, v)]
    rows = torch.nn.functional.pad(q.float(), (0, 0, 0, nq * block_q - tq)).view(b * h * nq, block_q, d)
    key = at.unsqueeze(-1) * block_k + torch.arange(block_k, device="cuda")
    seen = (((blocks >= 0) & (blocks < nk)).unsqueeze(-1) & (key < k_lens.view(b, 1, 1, 1, 1))).view(b * h * nq, 1, -1)
    score = torch.bmm(rows, gathered[0].transpose(1, 2)).mul_(s["scale"]).masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.bmm(p, gathered[1]) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log()).view(b, h, nq * block_q)[:, :, :tq]
    out = out.view(b, h, nq * block_q, d)[:, :, :tq].permute(0, 2, 1, 3)
    row = torch.arange(tq, device="cuda") < q_lens.view(b, 1)   # rows behind a sequence's end stay as they were
    return {"out": torch.where(row.view(b, tq, 1, 1), out.bfloat16(), s["out"]), "lse": torch.where(row.view(b, 1, tq), lse, s["lse"])}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return {n: _rope_exact(s, s[n], s["gamma_" + n]) for n in ("q", "k")}
    if case["kind"] == "select":
        return _select_exact(s, _lens(case) if case["ragged"] else [(case["tokens_q"], case["tokens_k"])] * case["batch"])
    b, h, tq, d = s["q"].shape
    hk, tk = s["k"].shape[1:3]
    nq, share = -(-tq // case["block_q"]), h // hk
    out, lse = torch.zeros(b, tq, h, d, dtype=torch.float64, device="cuda"), torch.zeros(b, h, tq, dtype=torch.float64, device="cuda")
    lens = _lens(case) if case["ragged"] else [(tq, tk)] * b
    offset = torch.arange(case["block_k"], device="cuda")
    for i, (nqt, nkt) in enumerate(lens):
        for j in range(h):
            keys, values = (s[n][i, j // share].double() for n in ("k", "v"))
            query = torch.zeros(nq * case["block_q"], d, dtype=torch.float64, device="cuda")
            query[:tq] = s["q"][i, j].double()
            if s["blocks"] is None:
                weight = query @ keys[:nkt].T * s["scale"]
                total = torch.logsumexp(weight, -1)
                got = torch.softmax(weight, -1) @ values[:nkt]
            else:
                index = s["blocks"][i, j].long().unsqueeze(-1) * case["block_k"] + offset
                index = index.view(nq, -1)
                out_of = (index < 0) | (index >= nkt)
                index = index.clamp(0, tk - 1)
                weight = torch.matmul(query.view(nq, -1, d), keys[index].transpose(1, 2).contiguous()) * s["scale"]
                weight = weight.masked_fill(out_of.unsqueeze(1), -math.inf)
                total = torch.logsumexp(weight, -1).reshape(-1)
                got = torch.nan_to_num(torch.matmul(torch.softmax(weight, -1), values[index])).view(-1, d)
            out[i, :nqt, j], lse[i, j, :nqt] = got[:nqt], total[:nqt]
    return {"out": out, "lse": lse}


def _rope_exact(s, x, gamma):
    x = x.double()
    y = gamma.double() * x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + 1e-6)
    at, pairs = 0, sum(s["axis_pairs"])
    out = y.clone()
    for axis, n in enumerate(s["axis_pairs"]):
        angle = s["positions"][:, :, axis].double().unsqueeze(1).unsqueeze(-1) * s["freqs"][at:at + n]
        turn = torch.polar(torch.ones_like(angle), angle)
        p = torch.arange(at, at + n, device="cuda")
        first, second = (p, p + pairs) if s["halves"] else (2 * p, 2 * p + 1)
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        out[..., first], out[..., second] = z.real, z.imag
        at += n
    return out


def _select_exact(s, lens):
    (b, h, tq, d), block_q, block_k, top = s["q"].shape, s["block_q"], s["block_k"], s["top"]
    blocks = torch.full((b, h, -(-tq // block_q), top), -1, dtype=torch.int32, device="cuda")
    scores = torch.full(blocks.shape, math.nan, dtype=torch.float64, device="cuda")
    for i, (nqt, nkt) in enumerate(lens):
        sums = []
        for x, n, block in ((s["q"][i], nqt, block_q), (s["k"][i], nkt, block_k)):
            owner = torch.arange(n, device="cuda") // block
            total = torch.zeros(h, -(-n // block), d, dtype=torch.float64, device="cuda").index_add_(1, owner, x[:, :n].double())
            sums.append(total / torch.bincount(owner).view(1, -1, 1))
        score = torch.matmul(sums[0], sums[1].transpose(1, 2).contiguous())
        kept = min(top, score.shape[-1])
        best = (-score).sort(dim=-1, stable=True).indices[..., :kept].sort(-1).values
        blocks[i, :, :score.shape[1], :kept] = best.int()
        scores[i, :, :score.shape[1], :kept] = score.gather(-1, best)
    return {"blocks": blocks, "scores": scores}
