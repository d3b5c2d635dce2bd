"""What the attention path's entry points refuse, before any GPU work: no device is needed (pointers are host buffers that are
never dereferenced), and what the binding refuses to hand on."""

import ctypes

import pytest
import torch

import paper_2603_02883_amd as F
from paper_2603_02883_amd import binding as B

P = ctypes.c_void_p
BUF = ctypes.create_string_buffer(4096 + 64)
AL = (ctypes.addressof(BUF) + 63) // 64 * 64
NAN, INF = float("nan"), float("inf")


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


def rope(q=P(AL), sq=strides(2048, 64, 256), k=P(AL), sk=strides(2048, 64, 256), batch=2, tokens=4, hq=2, hk=2, dim=64, norm=1, gq=None, gk=None,
         eps=1e-6, pos=P(AL), shared=0, freqs=P(AL), pairs=(8, 24), axes=None, pairing=0, qo=P(AL), ko=P(AL)):
    p = (ctypes.c_int32 * max(len(pairs), 1))(*pairs) if pairs is not None else None
    return B.lib().fb4_qk_norm_rope(q, sq, k, sk, batch, tokens, hq, hk, dim, norm, gq, gk, eps, pos, shared, freqs, p,
                                    len(pairs) if axes is None else axes, pairing, qo, ko, None)


def test_rope_refusals():
    assert rope(batch=0) == F.OK and rope(tokens=0, q=None, k=None) == F.OK
    for bad in (dict(batch=-1), dict(tokens=-1), dict(hq=0), dict(hk=-1), dict(dim=0), dict(norm=2), dict(eps=-1.0), dict(eps=NAN), dict(shared=2),
                dict(pairing=2), dict(pairs=(), axes=-1), dict(pairs=(0, 8)), dict(pairs=(16, 17)), dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1)),
                dict(pairs=None, axes=1), dict(q=None), dict(k=None), dict(sq=None), dict(sk=None), dict(qo=None), dict(ko=None), dict(pos=None),
                dict(freqs=None), dict(sq=strides(-8, 64, 256))):
        assert rope(**bad) == F.ERR_INVALID_ARG, bad
    for bad in (dict(dim=60, pairs=(8,)), dict(dim=264), dict(pairs=(6, 8), pairing=1), dict(pairs=(4,) * 5), dict(sq=strides(2048, 60, 256)),
                dict(sk=strides(2048, 64, 2 ** 36)), dict(q=P(AL + 8)), dict(k=P(AL + 2)), dict(qo=P(AL + 8)), dict(ko=P(AL + 4)), dict(gq=P(AL + 2)),
                dict(pos=P(AL + 2)), dict(freqs=P(AL + 4)), dict(tokens=2 ** 25), dict(batch=2 ** 62, tokens=2 ** 62), dict(hq=70000)):
        assert rope(**bad) == F.ERR_UNSUPPORTED, bad


def select(q=P(AL), k=P(AL), batch=1, heads=4, hk=2, tq=200, tk=300, dim=64, lens=None, bq=64, bk=128, top=2, blocks=P(AL), scores=None, ws=P(AL),
           size=1 << 20):
    return B.lib().fb4_select_key_blocks(q, k, batch, heads, hk, tq, tk, dim, lens, bq, bk, top, blocks, scores, ws, size, None)


def test_select_refusals():
    assert select(batch=0) == F.OK and select(tq=0) == F.OK and select(top=0, blocks=None) == F.OK
    size = B.lib().fb4_select_key_blocks_workspace(1, 4, 2, 200, 300, 64, 64, 128)
    assert size == (4 * 4 + 2 * 3) * 64 * 8
    for bad in (dict(batch=-1), dict(heads=0), dict(hk=0), dict(hk=3), dict(tq=-1), dict(tk=-1), dict(dim=0), dict(top=-1), dict(q=None), dict(k=None),
                dict(blocks=None), dict(ws=None), dict(size=size - 1)):
        assert select(**bad) == F.ERR_INVALID_ARG, bad
    for bad in (dict(dim=60), dict(dim=136), dict(bq=32), dict(bk=96), dict(bk=0), dict(q=P(AL + 8)), dict(k=P(AL + 8)), dict(lens=P(AL + 2)),
                dict(blocks=P(AL + 1)), dict(scores=P(AL + 2)), dict(ws=P(AL + 4)), dict(tk=128 * 2049, size=1 << 40), dict(heads=70000, hk=1),
                dict(tq=2 ** 31), dict(tk=2 ** 31), dict(batch=2 ** 32)):
        assert select(**bad) == F.ERR_UNSUPPORTED, bad
    assert B.lib().fb4_select_key_blocks_workspace(1, 4, 3, 200, 300, 64, 64, 128) == 0


def attention(q=P(AL), k=P(AL), v=P(AL), sv=strides(0, 64, 128), batch=1, heads=4, hk=2, tq=200, tk=300, dim=64, lens=None, blocks=P(AL), top=2, bq=64,
              bk=128, scale=0.125, out=P(AL), so=strides(0, 64, 256), lse=None, ws=None, size=0):
    return B.lib().fb4_block_attention(q, k, v, sv, batch, heads, hk, tq, tk, dim, lens, blocks, top, bq, bk, scale, out, so, lse, ws, size, None)


def test_attention_refusals():
    assert attention(batch=0) == F.OK and attention(tq=0, out=None) == F.OK
    big = dict(ws=P(AL), size=1 << 40)   # (enough for any of these)
    for bad in (dict(batch=-1), dict(heads=0), dict(hk=0), dict(hk=3), dict(tq=-1), dict(tk=-1), dict(dim=0), dict(top=-2), dict(q=None), dict(k=None),
                dict(v=None), dict(blocks=None), dict(top=-1), dict(sv=None), dict(out=None), dict(so=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF),
                dict(sv=strides(0, -8, 128)), dict(so=strides(0, 64, -8))):
        assert attention(**{**big, **bad}) == F.ERR_INVALID_ARG, bad
    for bad in (dict(dim=60), dict(dim=136), dict(bq=32), dict(bk=96), dict(bk=0), dict(q=P(AL + 8)), dict(k=P(AL + 8)), dict(v=P(AL + 8)),
                dict(out=P(AL + 8)), dict(lens=P(AL + 2)), dict(blocks=P(AL + 1)), dict(lse=P(AL + 2)), dict(sv=strides(0, 64, 132)),
                dict(so=strides(4, 64, 256)), dict(sv=strides(0, 64, 2 ** 25)), dict(heads=70000, hk=1), dict(tq=2 ** 31), dict(batch=2 ** 24)):
        assert attention(**{**big, **bad}) == F.ERR_UNSUPPORTED, bad
    # a workspace that is too small, or none where there has to be one
    need = B.lib().fb4_block_attention_workspace(1, 1, 1, 1, 1 << 20, 64, -1, 64, 64)
    one = dict(heads=1, hk=1, tq=1, tk=1 << 20, blocks=None, top=-1, bk=64)
    if need:
        assert attention(**one, ws=P(AL), size=need - 1) == F.ERR_INVALID_ARG
        assert attention(**one, ws=None, size=need) == F.ERR_INVALID_ARG
        assert attention(**one, ws=P(AL + 4), size=need) == F.ERR_UNSUPPORTED
    assert B.lib().fb4_block_attention_workspace(1, 4, 3, 1, 1 << 20, 64, -1, 64, 64) == 0


def test_binding_hands_on_no_host_tensors_and_no_other_types():
    """A host pointer or another type's would be read as the device's bf16."""
    q = torch.zeros((1, 2, 4, 8), dtype=torch.bfloat16)
    for call in (lambda: F.fb4_qk_norm_rope(q, q, None, None, ()), lambda: F.fb4_select_key_blocks(q, q, 1), lambda: F.fb4_block_attention(q, q, q)):
        with pytest.raises(F.Fb4Error) as e:
            call()
        assert e.value.code == F.ERR_INVALID_ARG


def test_empty_calls_need_no_pointers_in_the_binding_either():
    assert F.strerror(F.OK) and B.lib().fb4_block_attention_workspace(0, 1, 1, 0, 0, 8, 0, 64, 64) == 0


class OnGpu:
    """As much of a GPU tensor as the binding looks at before it hands it on."""
    is_cuda, device = True, "cuda:0"

    def __init__(self, *shape):
        self.shape = shape

    def dim(self):
        return len(self.shape)


def test_outputs_are_made_on_the_stream_that_the_call_runs_on(monkeypatch):
    """A fill, and whatever used the memory before, come before the kernels only on the kernels' own stream; the caller's may be far
    behind."""
    import contextlib
    from types import SimpleNamespace
    now, made, handed = ["callers"], [], []

    @contextlib.contextmanager
    def on(stream):
        now.append(stream.name)
        yield
        now.pop()

    def maker(kind):
        def make(shape, dtype, device):
            t = OnGpu(*(shape if isinstance(shape, tuple) else (shape,)))
            t.made, t.kept_for = (kind, now[-1]), []
            t.record_stream = t.kept_for.append
            made.append(t)
            return t
        return make

    def call(*args):
        handed.append(args)
        return F.OK
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch, "empty", maker("empty"))
    monkeypatch.setattr(torch, "zeros", maker("zeros"))
    monkeypatch.setattr(B, "_heads_call", SimpleNamespace(qk_norm_rope=call, select_key_blocks=call, block_attention=call))
    monkeypatch.setattr(B, "_get_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda device: 7)
    side = SimpleNamespace(name="side", cuda_stream=99)
    q, k, lens = OnGpu(2, 4, 100, 64), OnGpu(2, 2, 300, 64), OnGpu(2, 2)
    calls = [lambda s: F.fb4_qk_norm_rope(q, k, None, None, (), stream=s), lambda s: F.fb4_select_key_blocks(q, k, 2, want_scores=True, stream=s),
             lambda s: F.fb4_block_attention(q, k, k, want_lse=True, stream=s), lambda s: F.fb4_block_attention(q, k, k, lens=lens, want_lse=True, stream=s)]
    for kind, one in zip(("empty", "empty", "empty", "zeros"), calls):
        for stream, name, handle in ((side, "side", 99), (None, "callers", 7)):
            made.clear()
            outs = one(stream)
            assert len(made) == 2 and all(a is b for a, b in zip(outs, made)) and handed[-1][-1] == handle
            assert all(t.made == (kind, name) for t in made), [t.made for t in made]
            # (the memory comes back only when the caller's stream, where the results are used, is done with it too)
            assert all(t.kept_for == ([] if stream is None else ["callers"]) for t in made)


def test_select_refuses_launches_of_more_than_32_bits_of_threads():
    """Both kernels' launches have to fit before the first runs: the choice takes 512 threads per 16 blocks of queries of a head, 1024
    per 32 with 513 to 1024 blocks of keys."""
    big = dict(ws=P(AL), size=1 << 50, dim=8, bk=64)
    many = dict(heads=60000, hk=1, tq=1, **big)
    for bad in (dict(batch=140, tk=1), dict(batch=150, tk=1), dict(batch=70, tk=64 * 513), dict(batch=70, tk=64 * 1024)):
        assert select(**{**many, **bad}) == F.ERR_UNSUPPORTED, bad
    # what fits comes as far as the device
    if not torch.cuda.is_available():
        for good in (dict(batch=139, tk=1), dict(batch=69, tk=64 * 1024), dict(batch=70, tk=64 * 512), dict(batch=100, tk=64 * 1025)):
            assert select(**{**many, **good}) == F.ERR_HIP, good


def test_sizes_whose_products_pass_64_bits_are_refused():
    """Each size in its own range, their product a small number modulo 2^64: what a check of the wrapped product would let through."""
    lib = B.lib()
    for batch, heads, tq in ((2 ** 30, 2 ** 15, 2 ** 25), (2 ** 31 - 1, 2 ** 15, 2 ** 31 - 64), (2 ** 27, 2 ** 15, 2 ** 22 * 64), (2 ** 30, 2 ** 15, 2 ** 25 + 64)):
        sizes = dict(batch=batch, heads=heads, hk=1, tq=tq, tk=0, dim=64, bq=64, bk=64)
        assert select(**sizes, ws=P(AL), size=2 ** 64 - 1) == F.ERR_UNSUPPORTED, sizes
        assert attention(**sizes, ws=P(AL), size=2 ** 64 - 1) == F.ERR_UNSUPPORTED, sizes
        assert lib.fb4_select_key_blocks_workspace(batch, heads, 1, tq, 0, 64, 64, 64) == 0
        assert lib.fb4_block_attention_workspace(batch, heads, 1, tq, 0, 64, 2, 64, 64) == 0
    assert select(batch=2 ** 31 - 1, heads=1, hk=1, tq=1, tk=2 ** 31 - 1, bk=64, ws=P(AL), size=2 ** 64 - 1) == F.ERR_UNSUPPORTED


class Laid(OnGpu):
    """... and as much as the calls through ctypes look at: a contiguous tensor of no memory."""

    def __init__(self, dtype, *shape):
        self.dtype, self.shape, self.device = dtype, torch.Size(shape), torch.device("cuda", 0)

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def stride(self, i):
        return self.shape[i + 1:].numel()

    def data_ptr(self):
        return AL

    def transpose(self, a, b):
        return self


def test_numbers_that_c_would_cut_off_are_refused(monkeypatch):
    """A block size of 2^32 + 64 is 64 to C, for which the list has too few rows."""
    class Library:
        fb4_select_key_blocks_workspace = fb4_block_attention_workspace = staticmethod(lambda *a: 0)
        fb4_strerror = staticmethod(lambda code: b"refused")

        def __getattr__(self, name):
            def call(*a):
                handed.append(name)
                return F.OK
            return call
    handed = []
    monkeypatch.setattr(B, "_lib", Library())
    bf, i32, far = torch.bfloat16, torch.int32, 2 ** 32
    q, k, ws = Laid(bf, 1, 2, 100, 64), Laid(bf, 1, 2, 100, 64), Laid(torch.uint8, 4096)

    def choose(bq=64, bk=64):
        return B.HeadsCall.select_key_blocks(q, k, 3, bq, bk, None, Laid(i32, 1, 2, -(-100 // bq), 3), None, ws, 0, None)

    def attend(bq=64, bk=64):
        return B.HeadsCall.block_attention(q, k, k, Laid(i32, 1, 2, -(-100 // bq), 3), 1.0, bq, bk, None, Laid(bf, 1, 100, 2, 64), None, ws, 0, None)

    def turn(pairs=(8, 8), pairing=0, q=q, k=k):
        return B.HeadsCall.qk_norm_rope(q, k, Laid(i32, 1, 100, len(pairs)), Laid(torch.float64, sum(pairs)), pairs, None, None, 1e-6, True, pairing,
                                        q, k, 0, None)
    assert choose() == attend() == turn() == F.OK and len(handed) == 3
    wide, seq = Laid(bf, 1, far + 2, 100, 64), Laid(bf, 1, 2, 100, 64)
    for call in (lambda: choose(far + 64), lambda: choose(64, far + 64), lambda: attend(far + 128), lambda: attend(64, far + 64),
                 lambda: turn((far + 8,)), lambda: turn((far + 4, 4 - far)), lambda: turn(pairing=far), lambda: turn(pairing=far + 1), lambda: turn(q=wide),
                 lambda: turn(q=seq, k=wide)):
        with pytest.raises(F.Fb4Error):
            call()
    assert len(handed) == 3


def test_scales_whose_product_with_log2_e_leaves_fp32_are_refused():
    assert attention(ws=P(AL), size=1 << 40, scale=3e38) == F.ERR_UNSUPPORTED
    assert attention(ws=P(AL), size=1 << 40, scale=2.0 ** 127 * 1.0001) == F.ERR_UNSUPPORTED
    if not torch.cuda.is_available():   # (as far as the device)
        assert attention(ws=P(AL), size=1 << 40, scale=2.0 ** 127) == F.ERR_HIP


def test_rotation_refuses_outputs_on_memory_that_is_read_elsewhere():
    """A row that is written while another workgroup still reads it.  In place, row upon row, is none; neither is a gap between rows."""
    n = 2 * 2 * 4 * 64 * 2                                  # bytes of [2][2][4][64]
    dense, packed, swapped = strides(512, 256, 64), strides(4 * 6 * 64, 64, 6 * 64), strides(64, 2 * 64, 4 * 64)
    far = P(AL + (1 << 30))
    served = F.ERR_HIP if not torch.cuda.is_available() else None
    base = dict(pairs=(8,), sq=dense, sk=dense, k=far, ko=P(AL + (1 << 31)))
    bad = [dict(sq=packed, qo=P(AL)), dict(sq=packed, qo=P(AL + 6 * 64 * 2 * 7)), dict(sq=swapped, qo=P(AL)), dict(qo=P(AL + 16)), dict(qo=P(AL + n - 16)),
           dict(q=P(AL + n - 16), qo=P(AL)), dict(k=P(AL), q=far, qo=P(AL)), dict(k=P(AL), q=far, sk=packed, ko=P(AL + 6 * 64 * 2)),
           dict(qo=far), dict(q=far, qo=P(AL + (1 << 32)), ko=P(AL + (1 << 32) + n - 16)),
           dict(q=P(AL), sq=strides(0, 0, 0), qo=P(AL)), dict(q=P(AL), sq=strides(8, 8, 8), qo=P(AL + 128))]
    good = [dict(qo=P(AL)), dict(qo=P(AL + n)), dict(q=P(AL + n), qo=P(AL)), dict(k=P(AL), q=far, qo=P(AL + n), ko=P(AL)),
            # one sequence of four tokens in its packed projection's last gap; all of an output between two sequences far apart
            dict(batch=1, hq=1, tokens=1, sq=packed, qo=P(AL + 128)), dict(sq=strides(1 << 20, 256, 64), qo=P(AL + 4096)),
            dict(q=P(AL), sq=strides(0, 0, 0), qo=P(AL + 128)), dict(hk=0, k=None, ko=None, qo=P(AL)), dict(k=P(AL + n), sk=strides(0, 0, 64), qo=P(AL + 2 * n))]
    for case in bad:
        assert rope(**{**base, "qo": P(AL + (1 << 33)), **case}) == F.ERR_INVALID_ARG, case
    if served is not None:                                  # (as far as the device)
        for case in good:
            assert rope(**{**base, "qo": P(AL + (1 << 33)), **case}) == served, case
