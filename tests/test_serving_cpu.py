"""What the serving entry points refuse, before any GPU work: no device is needed (pointers are host buffers that are never
dereferenced), and what the binding refuses to hand on."""

import ctypes

import pytest
import torch

import paper_2603_02883_amd as F
from paper_2603_02883_amd import binding as B

P = ctypes.c_void_p
BUF = ctypes.create_string_buffer(4096 + 64)
AL = (ctypes.addressof(BUF) + 63) // 64 * 64
NAN, INF = float("nan"), float("inf")
SERVED = F.ERR_HIP if not torch.cuda.is_available() else None   # (as far as the device)


def strides(*s):
    return (ctypes.c_int64 * 2)(*s)


def plan(lens=P(AL), adds=P(AL), batch=3, page=16, tables=P(AL), wide=4, free=P(AL), n_free=9, count=P(AL), lens_out=P(AL), count_out=P(AL), starts=P(AL),
         slots=P(AL), positions=P(AL), tokens=7):
    return B.lib().fb4_cache_plan(lens, adds, batch, page, tables, wide, free, n_free, count, lens_out, count_out, starts, slots, positions, tokens, None)


def test_plan_refusals():
    for bad in (dict(batch=-1), dict(wide=-1), dict(n_free=-1), dict(tokens=-1), dict(lens=None), dict(adds=None), dict(tables=None), dict(free=None),
                dict(count=None), dict(lens_out=None), dict(count_out=None), dict(starts=None), dict(slots=None)):
        assert plan(**bad) == F.ERR_INVALID_ARG, bad
    for bad in (dict(page=0), dict(page=-16), dict(page=48), dict(page=256), dict(batch=4097), dict(wide=2 ** 27), dict(batch=4096, wide=2 ** 19), dict(n_free=2 ** 31),
                dict(tokens=2 ** 31), dict(lens=P(AL + 2)), dict(adds=P(AL + 1)), dict(tables=P(AL + 2)), dict(free=P(AL + 2)), dict(count=P(AL + 2)),
                dict(lens_out=P(AL + 2)), dict(count_out=P(AL + 2)), dict(starts=P(AL + 2)), dict(slots=P(AL + 2)), dict(positions=P(AL + 2)),
                dict(batch=2 ** 62), dict(wide=2 ** 62)):
        assert plan(**bad) == F.ERR_UNSUPPORTED, bad
    if SERVED is not None:
        for good in (dict(), dict(positions=None), dict(tokens=0, slots=None), dict(batch=0, lens=None, adds=None, lens_out=None, tables=None), dict(n_free=0, free=None),
                     dict(batch=4096, wide=2 ** 19 - 1)):
            assert plan(**good) == SERVED, good


def store(k=P(AL), sk=strides(64, 128), v=P(AL), sv=strides(64, 128), tokens=5, heads=2, dim=64, slots=P(AL), cache=P(AL), scales=P(AL), pages=4, page=16):
    return B.lib().fb4_cache_store(k, sk, v, sv, tokens, heads, dim, slots, cache, scales, pages, page, None)


def test_store_refusals():
    assert store(tokens=0, k=None) == F.OK and store(pages=0, cache=None) == F.OK
    for bad in (dict(tokens=-1), dict(heads=0), dict(dim=0), dict(pages=-1), dict(k=None), dict(sk=None), dict(v=None), dict(sv=None), dict(slots=None), dict(cache=None),
                dict(scales=None), dict(sk=strides(-8, 128)), dict(sv=strides(64, -8))):
        assert store(**bad) == F.ERR_INVALID_ARG, bad
    for bad in (dict(dim=60), dict(dim=136), dict(heads=65536), dict(page=8), dict(page=17), dict(tokens=2 ** 31), dict(pages=2 ** 27), dict(k=P(AL + 8)), dict(v=P(AL + 2)),
                dict(slots=P(AL + 2)), dict(cache=P(AL + 8)), dict(sk=strides(60, 128)), dict(sv=strides(64, 2 ** 36)), dict(tokens=2 ** 30, heads=60000),
                dict(tokens=2 ** 62), dict(pages=2 ** 62)):
        assert store(**bad) == F.ERR_UNSUPPORTED, bad


def attend(q=P(AL), sq=strides(64, 256), tokens=3, heads=4, hk=2, dim=64, cache=P(AL), scales=P(AL), pages=9, page=16, tables=P(AL), wide=5, lens=P(AL), starts=P(AL),
           batch=2, causal=1, scale=0.125, out=P(AL), so=strides(64, 256), lse=None, ws=P(AL), size=1 << 40):
    return B.lib().fb4_cache_attention(q, sq, tokens, heads, hk, dim, cache, scales, pages, page, tables, wide, lens, starts, batch, causal, scale, out, so, lse, ws, size, None)


def test_attention_refusals():
    assert attend(tokens=0, q=None) == F.OK and attend(batch=0, out=None) == F.OK
    for bad in (dict(tokens=-1), dict(heads=0), dict(hk=0), dict(hk=3), dict(dim=0), dict(pages=-1), dict(wide=-1), dict(batch=-1), dict(causal=2), dict(causal=-1),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(q=None), dict(sq=None), dict(cache=None), dict(scales=None), dict(tables=None),
                dict(lens=None), dict(starts=None), dict(out=None), dict(so=None), dict(sq=strides(-8, 256)), dict(so=strides(64, -8))):
        assert attend(**bad) == F.ERR_INVALID_ARG, bad
    for bad in (dict(dim=60), dict(dim=136), dict(heads=70000, hk=1), dict(page=0), dict(page=24), dict(wide=2 ** 27), dict(pages=2 ** 27), dict(batch=4097),
                dict(tokens=2 ** 31), dict(tokens=2 ** 30, heads=4, hk=1), dict(scale=2.0 ** 127 * 1.0001), dict(q=P(AL + 8)), dict(cache=P(AL + 8)), dict(tables=P(AL + 2)),
                dict(lens=P(AL + 2)), dict(starts=P(AL + 2)), dict(out=P(AL + 8)), dict(lse=P(AL + 2)), dict(ws=P(AL + 4), wide=100), dict(sq=strides(4, 256)),
                dict(so=strides(64, 252)), dict(sq=strides(64, 2 ** 36)), dict(tokens=2 ** 62), dict(tokens=2 ** 30, heads=60000, hk=60000)):
        assert attend(**bad) == F.ERR_UNSUPPORTED, bad
    size = lambda **kw: B.lib().fb4_cache_attention_workspace(*{**dict(tokens=1, heads=4, hk=2, dim=64, page=16, wide=1000, batch=1), **kw}.values())
    need = size()
    assert need > 0 and size(wide=1) == 0 and size(tokens=1 << 20) == 0 and size(tokens=-1) == size(hk=3) == size(batch=4097) == size(page=20) == size(tokens=0) == 0
    one = dict(tokens=1, wide=1000, batch=1)
    assert attend(**one, size=need - 1) == F.ERR_INVALID_ARG and attend(**one, ws=None, size=need) == F.ERR_INVALID_ARG
    if SERVED is not None:
        for good in (dict(**one, size=need), dict(wide=0, tables=None, ws=None, size=0), dict(pages=0, cache=None, scales=None, tables=None), dict(scale=2.0 ** 127)):
            assert attend(**good) == SERVED, good


def test_matvec_refusals():
    call = lambda h=None, x=P(AL), rows=2, sx=64, codes=P(AL), meta=P(AL), n=5, cols=64, block=32, bias=None, out=P(AL), dtype=0, so=5: B.lib().fb4_matvec(
        h, x, rows, sx, codes, meta, n, cols, block, bias, out, dtype, so, None)
    assert call() == F.ERR_INVALID_ARG                                # (no handle; what is refused before it is looked into:)
    handle = ctypes.create_string_buffer(1 << 14)
    h = ctypes.addressof(handle)
    for ok in (dict(rows=0, x=None, out=None), dict(n=0, codes=None, out=None)):
        assert call(h, **ok) == F.OK, ok
    for bad in (dict(rows=-1), dict(n=-1), dict(cols=-32), dict(sx=63), dict(so=4), dict(block=8), dict(block=64), dict(dtype=2), dict(x=None), dict(codes=None), dict(meta=None),
                dict(out=None)):
        assert call(h, **bad) == F.ERR_INVALID_ARG, bad
    for bad in (dict(rows=65), dict(cols=48), dict(n=2 ** 28, so=2 ** 28), dict(cols=2 ** 25, sx=2 ** 25), dict(x=P(AL + 8)), dict(sx=68), dict(codes=P(AL + 8)), dict(meta=P(AL + 1)),
                dict(meta=P(AL + 2), block=16), dict(bias=P(AL + 2)), dict(out=P(AL + 1)), dict(out=P(AL + 2), dtype=1), dict(sx=2 ** 36), dict(rows=2 ** 62),
                dict(n=2 ** 62, so=2 ** 62), dict(cols=2 ** 62, sx=2 ** 62)):
        assert call(h, **bad) == F.ERR_UNSUPPORTED, bad


def test_binding_hands_on_no_host_tensors():
    x, i = torch.zeros((2, 4, 32), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    u = torch.zeros((2, 4, 2, 16 * 32), dtype=torch.uint8)
    luts = F.Luts(None, 32)
    for call in (lambda: F.fb4_matvec(luts, x[0], u[0, 0], i), lambda: F.fb4_cache_plan(i, i, i.view(2, 1), i, i[:1], 16, 2),
                 lambda: F.fb4_cache_store(x, x, i, u, u[..., 0], 16), lambda: F.fb4_cache_attention(x, u, u[..., 0], i.view(2, 1), i, i, 16)):
        with pytest.raises(F.Fb4Error) as e:
            call()
        assert e.value.code == F.ERR_INVALID_ARG


class Laid:
    """As much of a contiguous GPU tensor as the binding and the calls through ctypes look at, of no memory."""
    is_cuda = True

    def __init__(self, dtype, *shape, device=0, dense=True, inner=1):
        self.dtype, self.shape, self.device, self.dense, self.inner = dtype, torch.Size(shape), torch.device("cuda", device), dense, inner

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return self.dense

    def numel(self):
        return self.shape.numel()

    def stride(self, i):
        return self.shape[i + 1:].numel() if i + 1 < len(self.shape) else self.inner

    def data_ptr(self):
        return AL

    def transpose(self, a, b):
        return self


BF, I32, U8, F32, FAR = torch.bfloat16, torch.int32, torch.uint8, torch.float32, 2 ** 32


@pytest.fixture
def handed(monkeypatch):
    """The library's calls, noted and not made."""
    class Library:
        fb4_cache_attention_workspace = staticmethod(lambda *a: 0)
        fb4_strerror = staticmethod(lambda code: b"refused")

        def __getattr__(self, name):
            def call(*a):
                seen.append(name)
                return F.OK
            return call
    seen = []
    monkeypatch.setattr(B, "_lib", Library())
    return seen


def refused(call, code=None):
    with pytest.raises(F.Fb4Error) as e:
        call()
    assert code is None or e.value.code == code


def test_shapes_types_devices_and_numbers_that_c_would_cut_off(handed):
    S = B.ServingCall

    def matvec(x=Laid(BF, 3, 64), codes=Laid(U8, 5, 32), meta=Laid(torch.int16, 5, 2), block=32, bias=Laid(F32, 5), out=Laid(BF, 3, 5)):
        return S.matvec(None, x, codes, meta, block, bias, out, 0, None)

    def plan_(lens=Laid(I32, 4), adds=Laid(I32, 4), tables=Laid(I32, 4, 3), free=Laid(I32, 9), count=Laid(I32, 1), page=16, lens_out=Laid(I32, 4), count_out=Laid(I32, 1),
              starts=Laid(I32, 5), slots=Laid(I32, 7), positions=Laid(I32, 7)):
        return S.cache_plan(lens, adds, tables, free, count, page, lens_out, count_out, starts, slots, positions, 0, None)

    def store_(k=Laid(BF, 2, 5, 64), v=Laid(BF, 2, 5, 64), slots=Laid(I32, 5), cache=Laid(U8, 2, 9, 2, 1024), scales=Laid(U8, 2, 9, 2), page=16):
        return S.cache_store(k, v, slots, cache, scales, page, 0, None)

    def attend_(q=Laid(BF, 4, 5, 64), cache=Laid(U8, 2, 9, 2, 1024), scales=Laid(U8, 2, 9, 2), tables=Laid(I32, 3, 4), lens=Laid(I32, 3), starts=Laid(I32, 4), page=16,
                out=Laid(BF, 5, 4, 64), lse=Laid(F32, 5, 4), ws=None):
        return S.cache_attention(q, cache, scales, tables, lens, starts, page, 1.0, True, out, lse, ws, 0, None)
    calls = (matvec, plan_, store_, attend_)
    assert all(c() == F.OK for c in calls) and len(handed) == 4
    assert matvec(bias=None) == plan_(positions=None) == attend_(lse=None) == F.OK and len(handed) == 7
    bad = {matvec: dict(x=[Laid(F32, 3, 64), Laid(BF, 3, 64, device=1), Laid(BF, 3, 64, inner=2), Laid(BF, 192), Laid(BF, 3, 96)], codes=[Laid(U8, 5, 31), Laid(U8, 5, 32, dense=False)],
                        meta=[Laid(torch.int16, 5, 4), Laid(I32, 5, 2), Laid(torch.int16, 4, 2)], block=[16, 0, FAR + 32], bias=[Laid(F32, 4), Laid(BF, 5)],
                        out=[Laid(BF, 3, 4), Laid(torch.float16, 3, 5), Laid(BF, 3, 5, device=1), Laid(BF, 3, 5, inner=2)]),
           plan_: dict(lens=[Laid(I32, 3), Laid(torch.int64, 4)], adds=[Laid(I32, 5)], tables=[Laid(I32, 12), Laid(I32, 4, 3, dense=False)], free=[Laid(I32, 3, 3)],
                       count=[Laid(I32, 2)], page=[0, FAR + 16], lens_out=[Laid(I32, 3)], count_out=[Laid(I32, 0)], starts=[Laid(I32, 4)], positions=[Laid(I32, 6)],
                       slots=[Laid(I32, 7, 1), Laid(torch.int64, 7)]),
           store_: dict(k=[Laid(BF, 2, 4, 64), Laid(F32, 2, 5, 64), Laid(BF, 3, 5, 64), Laid(BF, 2, 5, 64, inner=2)], v=[Laid(BF, 2, 5, 32), Laid(BF, 2, 5, 64, inner=2)],
                        slots=[Laid(I32, 4), Laid(I32, 5, dense=False)], cache=[Laid(U8, 2, 8, 2, 1024), Laid(U8, 2, 9, 2, 1024, dense=False), Laid(U8, 2, 9, 2, 512)],
                        scales=[Laid(U8, 2, 9), Laid(U8, 1, 9, 2), Laid(F32, 2, 9, 2)], page=[32, 0, FAR + 16]),
           attend_: dict(q=[Laid(BF, 4, 5, 32), Laid(BF, 4, 5, 64, inner=2), Laid(BF, 20, 64), Laid(BF, FAR + 4, 5, 64)], cache=[Laid(U8, 2, 9, 1, 1024)], scales=[Laid(U8, 9, 2)],
                         tables=[Laid(I32, 12), Laid(I32, 3, 4, dense=False)], lens=[Laid(I32, 4)], starts=[Laid(I32, 3)], page=[32, FAR + 16], out=[Laid(BF, 4, 5, 64)],
                         lse=[Laid(F32, 4, 5)], ws=[Laid(F32, 4)])}
    for call, arguments in bad.items():
        for name, values in arguments.items():
            for value in values:
                refused(lambda: call(**{name: value}))
    assert len(handed) == 7


def test_outputs_are_made_on_the_stream_that_the_call_runs_on(monkeypatch):
    import contextlib
    from types import SimpleNamespace
    now, made = ["callers"], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream.name)
        yield
        now.pop()

    def maker(kind):
        def make(shape, dtype, device):
            t = Laid(dtype, *(shape if isinstance(shape, tuple) else (shape,)))
            t.made, t.kept_for = (kind, now[-1]), []
            t.record_stream = t.kept_for.append
            made.append(t)
            return t
        return make

    def call(*args):
        handles.append(args[-1])
        return F.OK
    handles = []
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch, "empty", maker("empty"))
    monkeypatch.setattr(torch, "zeros", maker("zeros"))
    monkeypatch.setattr(B, "_serving_call", SimpleNamespace(matvec=call, cache_plan=call, cache_store=call, cache_attention=call))
    monkeypatch.setattr(B, "_get_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 7)
    side = SimpleNamespace(name="side", cuda_stream=99)
    luts, i4, table = F.Luts(None, 32), Laid(I32, 4), Laid(I32, 4, 3)
    calls = ((1, "empty", lambda s: F.fb4_matvec(luts, Laid(BF, 3, 64), Laid(U8, 5, 32), Laid(torch.int16, 5, 2), stream=s)),
             (5, "empty", lambda s: F.fb4_cache_plan(i4, i4, table, Laid(I32, 9), Laid(I32, 1), 16, 7, stream=s)),
             (0, "", lambda s: F.fb4_cache_store(Laid(BF, 2, 5, 64), None, None, None, None, 16, stream=s)),
             (2, "zeros", lambda s: F.fb4_cache_attention(Laid(BF, 4, 5, 64), None, None, None, None, None, 16, want_lse=True, stream=s)))
    for n, kind, one in calls:
        for stream, name, handle in ((side, "side", 99), (None, "callers", 7)):
            made.clear()
            one(stream)
            assert len(made) == n and handles[-1] == handle and all(t.made == (kind, name) for t in made)
            assert all(t.kept_for == ([] if stream is None else ["callers"]) for t in made)


@pytest.fixture(scope="module")
def shares(tmp_path_factory):
    """The attention's rules for its parts, compiled for the host with multiplications and additions fused and not."""
    import os
    import shutil
    import subprocess

    from paper_2603_02883_amd import build
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if shutil.which(hipcc) is None:
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("shares")
    (at / "shares.hip").write_text('#include "%s/fb4_cache_attention.hpp"\n' % build.CSRC + """
extern "C" unsigned share(unsigned long long sum, unsigned tiles, unsigned heads_k, unsigned rows) { return fb4::share_of_tiles(sum, tiles, heads_k, rows); }
extern "C" unsigned parts(unsigned len, unsigned share, unsigned rows) { return fb4::parts_of(len, share, rows); }
""")
    libs = []
    for mode in ("off", "fast-honor-pragmas"):
        lib = str(at / (mode + ".so"))
        subprocess.run([hipcc, "--offload-host-only", "-O2", "-std=c++17", "-mfma", "-ffp-contract=" + mode, "-fPIC", "-shared", str(at / "shares.hip"), "-o", lib], check=True,
                       capture_output=True)
        libs.append(ctypes.CDLL(lib))
        libs[-1].share.argtypes = [ctypes.c_ulonglong] + [ctypes.c_uint] * 3
        libs[-1].parts.argtypes = [ctypes.c_uint] * 3
        libs[-1].share.restype = libs[-1].parts.restype = ctypes.c_uint
    return libs


def test_both_launches_come_to_the_same_parts(shares):
    """The attention's launch and the joining one each compute the parts, in kernels that a compiler may treat apart: where two numbers of parts
    cost nearly the same the choice hangs on no rounding."""
    plain, fused = shares
    near = 0
    for n in range(1, 769):
        costs = [(p, -(-n * p // 512) * (1.2 if n * p > 256 else 1.0), 12 + n * p / 256 if p > 1 else 0.0) for p in range(1, 17) if p == 1 or n * p <= 1536]
        for i, (p, a, c) in enumerate(costs):
            for q, b, d in costs[i + 1:]:
                if a / p == b / q:
                    continue
                steps = (d - c + 6 * b - 6 * a) / (a / p - b / q)      # where p and q parts cost alike
                if 1 < steps < 2 ** 21:
                    for total in range(max(1, int(steps * n) - 1), int(steps * n) + 3):
                        near += 1
                        assert plain.share(total, n, 1, 128) == fused.share(total, n, 1, 128), (n, total)
    assert near > 10000


def test_parts_fit_their_workspace(shares):
    """All tiles' parts together are no more than the positions that the workspace and the launch have, whatever the sequences' lengths."""
    import random
    r, split = random.Random(5), 0
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))
    for _ in range(3000):
        batch, heads_k, group, page = log(1, 300), r.choice([1, 2, 8, 24]), r.choice([1, 3, 5]), 64
        wide = log(17, 40000)
        counts = [r.choice([1, 1, 0, log(1, 300), log(1, 3000)]) if r.random() < 0.9 else log(1, 9000) for _ in range(batch)] if r.random() < 0.7 else [log(1, 4000)] * batch
        lens = [r.choice([wide * page, log(1, wide * page), 0, 1, 64]) for _ in range(batch)] if r.random() < 0.8 else [wide * page] * batch
        tokens, dim = sum(counts) + r.choice([0, 5]), 8
        size = B.lib().fb4_cache_attention_workspace(tokens, heads_k * group, heads_k, dim, page, wide, batch)
        if not size:
            continue
        split += 1
        rows = 128 if tokens * group > 40 * batch or tokens * group >= 16384 + batch * group else 16
        positions = size // (rows * (dim + 2) * 4)
        tiles = [-(-n * group // rows) for n in counts]
        steps = [-(-n // 64) for n in lens]
        share = shares[0].share(sum(t * s for t, s in zip(tiles, steps)), sum(tiles), heads_k, rows)
        used = sum(t * shares[0].parts(n, share, rows) for t, n in zip(tiles, lens)) * heads_k
        assert used <= positions, (counts, lens, share)
    assert split > 300


def test_products_of_too_many_threads_are_refused():
    """Two tiles of sixteen rows of weights to a workgroup of 512: from 2^28 - 31 rows on a launch would have 2^32 threads."""
    handle = ctypes.create_string_buffer(1 << 14)
    call = lambda rows, n: B.lib().fb4_matvec(ctypes.addressof(handle), P(AL), rows, 1024, P(AL), P(AL), n, 1024, 32, None, P(AL + (1 << 45)), 0, n, None)
    for rows in (1, 33, 64):
        for n in (2 ** 28 - 31, 2 ** 28 - 1):
            assert call(rows, n) == F.ERR_UNSUPPORTED, (rows, n)
        if SERVED is not None:
            assert call(rows, 2 ** 28 - 32) == SERVED


def test_products_refuse_results_on_memory_that_is_read():
    """Rows of x between the results' rows, and the other way round, are beside them; one shared byte is not."""
    handle = ctypes.create_string_buffer(1 << 14)
    gig = lambda i: P(AL + (i << 30))
    call = lambda x=gig(0), sx=64, codes=gig(1), meta=gig(2), bias=gig(3), out=gig(4), so=48, rows=5, n=48, cols=64, dtype=0, block=32: B.lib().fb4_matvec(
        ctypes.addressof(handle), x, rows, sx, codes, meta, n, cols, block, bias, out, dtype, so, None)
    at = lambda i, b: P(AL + (i << 30) + b)
    bad = [dict(out=gig(0)), dict(out=gig(1)), dict(out=gig(2)), dict(out=gig(3)), dict(out=at(0, 4 * 128 + 126)), dict(out=at(0, -4 * 96 - 2)), dict(out=at(1, 48 * 32 - 2)),
           dict(out=at(2, 48 * 2 * 2 - 2)), dict(out=at(3, 48 * 4 - 2)), dict(out=at(3, -96 * 5 + 2)), dict(out=at(1, -100), so=200), dict(out=at(2, 48 * 4 * 2 - 4), dtype=1, block=16),
           dict(out=at(0, -5 * 192 + 4), dtype=1), dict(sx=128, so=128, out=at(0, 126)), dict(sx=128, so=128, out=at(0, 128 + 34)), dict(sx=128, so=128, out=at(0, -94)),
           dict(sx=128, so=64, dtype=1, n=32, out=at(0, 132)), dict(sx=64, so=1 << 20, out=at(0, 500)), dict(rows=1, sx=1 << 30, out=at(0, 126)), dict(sx=1 << 20, out=at(0, (4 << 21) + 64))]
    good = [dict(), dict(out=at(0, 5 * 128)), dict(out=at(0, -5 * 96)), dict(out=at(1, 48 * 32)), dict(out=at(2, 48 * 4)), dict(out=at(3, 48 * 4)), dict(out=gig(3), bias=None),
            dict(sx=128, so=128, out=at(0, 128)), dict(sx=128, so=128, out=at(0, -96)), dict(sx=128, so=128, out=at(0, 128 + 32)), dict(sx=128, so=64, dtype=1, n=32, out=at(0, 128)),
            dict(rows=1, sx=1 << 30, out=at(0, 128)), dict(sx=1 << 20, out=at(0, 3 << 20)), dict(cols=0, sx=0, out=gig(0), codes=gig(0), meta=gig(0))]
    for case in bad:
        assert call(**case) == F.ERR_INVALID_ARG, case
    assert call(so=(1 << 40) + 1) == F.ERR_UNSUPPORTED
    if SERVED is not None:
        for case in good:
            assert call(**case) == SERVED, case


def test_stores_refuse_inputs_on_memory_that_is_written():
    """[heads 2][tokens 5][64] rows, 4 pages of 16: a cache of 2 * 4 * 2 * 1024 bytes and 16 scales."""
    at = lambda i, b=0: P(AL + (i << 30) + b)
    n = 2 * 4 * 2 * 1024
    base = dict(k=at(0), v=at(1), slots=at(2), cache=at(3), scales=at(4))
    bad = [dict(k=at(3)), dict(v=at(3)), dict(slots=at(3)), dict(k=at(4, -16 + 16)), dict(v=at(4)), dict(slots=at(4, 12)), dict(scales=at(3)), dict(scales=at(3, n - 1)), dict(scales=at(3, -15)),
           dict(k=at(3, n - 16)), dict(v=at(3, -4 * 256 - 2 * 64 - 112)), dict(slots=at(3, -16)), dict(slots=at(4, -4 * 5 + 4)), dict(k=at(3, -1024 * 64), sk=strides(1 << 19, 1 << 13)),
           dict(v=at(4, -4 * 512), sv=strides(64, 256)), dict(scales=at(0, 191), sk=strides(0, 128 * 4), k=at(0, 64))]
    good = [dict(), dict(k=at(3, n)), dict(k=at(3, -5 * 256)), dict(v=at(4, 16)), dict(slots=at(3, -20)), dict(slots=at(4, 16)), dict(scales=at(3, n)), dict(scales=at(3, -16)), dict(v=at(0)),
            dict(scales=at(0, 256), sk=strides(64, 256)), dict(cache=at(0, 1 << 16), sk=strides(1 << 19, 64)),
            dict(scales=at(0, 192), sk=strides(0, 128 * 4), k=at(0, 64))]   # (behind a row of 128 bytes)
    for case in bad:
        assert store(**{**base, **case}) == F.ERR_INVALID_ARG, case
    if SERVED is not None:
        for case in good:
            assert store(**{**base, **case}) == SERVED, case


def test_products_of_no_channels_have_rows_without_a_place():
    """An empty tensor's rows lie one element apart: of no channels no stride counts."""
    x = torch.empty(4, 0, dtype=torch.bfloat16)
    handle = ctypes.create_string_buffer(1 << 14)
    call = lambda rows, stride: B.lib().fb4_matvec(ctypes.addressof(handle), None, rows, stride, None, None, 5, 0, 32, None, P(AL), 0, 5, None)
    assert x.stride(0) % 8
    if SERVED is not None:
        assert call(4, x.stride(0)) == call(1, 0) == call(4, 0) == call(4, 2 ** 50 + 1) == SERVED
    assert call(4, -1) == F.ERR_INVALID_ARG
