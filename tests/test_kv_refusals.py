"""What the key-value cache's calls refuse, without a GPU: the library before any CUDA call, the binding on fake tensors of a CUDA device."""
import ctypes
from ctypes import c_int32, c_int64, c_void_p

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2506_22694_b200 as vt
from paper_2506_22694_b200 import build as vt_build

pytestmark = pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
I32, I64, F32, BF16, E4M3, U8 = torch.int32, torch.int64, torch.float32, torch.bfloat16, torch.float8_e4m3fn, torch.uint8
OK, INVALID, WORKSPACE, UNSUPPORTED = 0, 1, 3, 6
P = 0x10000                                            # an address that is never looked at


class KV(ctypes.Structure):
    _fields_ = [("k", c_void_p), ("v", c_void_p), ("k_exp", c_void_p), ("v_exp", c_void_p), ("format", c_int32), ("n_pages", c_int32), ("heads", c_int32),
                ("page", c_int32), ("d", c_int32), ("stride_page", c_int64), ("stride_head", c_int64), ("stride_token", c_int64), ("pages", c_void_p),
                ("S", c_int32), ("max_pages", c_int32), ("pages_ld", c_int64)]


@pytest.fixture(scope="module")
def lib():
    vt_build.build()
    return vt.lib()


def cache(**kw):
    base = dict(k=P, v=P, k_exp=None, v_exp=None, format=0, n_pages=10, heads=8, page=16, d=128, stride_page=8 * 16 * 128, stride_head=16 * 128,
                stride_token=128, pages=P, S=2, max_pages=4, pages_ld=4)
    base.update(kw)
    return KV(**base)


BAD_CACHES = [dict(k=None), dict(v=None), dict(pages=None), dict(format=2), dict(format=-1), dict(k_exp=P), dict(v_exp=P), dict(format=1), dict(format=1, k_exp=P),
              dict(n_pages=0), dict(heads=0), dict(page=0), dict(S=-1), dict(max_pages=0), dict(pages_ld=3), dict(max_pages=2 ** 20, pages_ld=2 ** 20, page=2 ** 11),
              dict(stride_page=0), dict(stride_head=-128), dict(stride_token=132), dict(stride_token=0), dict(k=P + 8), dict(v=P + 2), dict(pages=P + 2),
              dict(format=1, k_exp=P + 8, v_exp=P), dict(format=1, k_exp=P, v_exp=P + 4), dict(format=1, k_exp=P, v_exp=P, stride_token=136)]


def test_workspace_sizes(lib):
    need = lambda **kw: vt.workspace_bytes(vt.VT_OP_KV_ATTEND, **kw)
    assert need(n=4, B=1, K=32, V=8, d=128) > 256 and need(n=0, B=1, K=8, V=8, d=64) > 256
    assert need(n=1, B=64, K=32, V=8, d=128) >= need(n=1, B=1, K=32, V=8, d=128)
    for bad in (dict(n=-1), dict(B=0), dict(B=65), dict(K=30), dict(K=4), dict(V=0), dict(d=80), dict(d=0), dict(d=512), dict(K=2048)):
        assert need(**{**dict(n=4, B=1, K=32, V=8, d=128), **bad}) == 0


def write(lib, c, **kw):
    a = dict(q=P, q_ld=1024, k=P, k_ld=1024, v=P, v_ld=1024, T=4, Hq=8, seq=None, index=P, positions=P, freqs=P, rot=128, interleaved=0, qw=None, kw=None,
             eps=1e-6, out=P, ws=None)
    a.update(kw)
    return lib.vt_qkv_write(a["q"], a["q_ld"], a["k"], a["k_ld"], a["v"], a["v_ld"], a["T"], a["Hq"], ctypes.byref(c) if c else None, a["seq"], a["index"],
                            a["positions"], a["freqs"], a["rot"], a["interleaved"], a["qw"], a["kw"], a["eps"], a["out"], a["ws"], None)


def read(lib, c, **kw):
    a = dict(seq=None, index=P, T=4, k=P, v=P, ws=None)
    a.update(kw)
    return lib.vt_kv_read(ctypes.byref(c) if c else None, a["seq"], a["index"], a["T"], a["k"], a["v"], a["ws"], None)


def attend(lib, c, **kw):
    a = dict(q=P, q_ld=32 * 128, Q=1, Hq=32, lens=P, node=None, parent=None, parent_ld=0, N=0, scale=0.1, out=P, lse=P, ws=P, ws_bytes=1 << 30)
    a.update(kw)
    return lib.vt_kv_attend(a["q"], a["q_ld"], a["Q"], a["Hq"], ctypes.byref(c) if c else None, a["lens"], a["node"], a["parent"], a["parent_ld"], a["N"],
                            a["scale"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


def commit(lib, c, **kw):
    a = dict(lens=P, path=P, n_accept=P, nodes=None, N=7, new_lens=P, ws=None)
    a.update(kw)
    return lib.vt_kv_commit(ctypes.byref(c) if c else None, a["lens"], a["path"], a["n_accept"], a["nodes"], a["N"], a["new_lens"], a["ws"], None)


@pytest.mark.parametrize("call", [write, read, attend, commit])
def test_a_cache_that_is_none(lib, call):
    assert call(lib, None) == INVALID
    for bad in BAD_CACHES:
        assert call(lib, cache(**bad)) == INVALID, bad
    for bad in (dict(d=80), dict(d=32), dict(d=512), dict(heads=2000)):
        assert call(lib, cache(**bad)) == UNSUPPORTED, bad


def test_write_refusals(lib):
    c = cache()
    for bad in (dict(T=-1), dict(Hq=-1), dict(Hq=2000), dict(Hq=0), dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(index=None), dict(positions=None),
                dict(freqs=None), dict(rot=0), dict(rot=8), dict(rot=144), dict(rot=-16), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(T=5),
                dict(k_ld=1016), dict(v_ld=8), dict(q_ld=1020), dict(q_ld=0), dict(k_ld=1028), dict(q=P + 2), dict(k=P + 8), dict(v=P + 4), dict(out=P + 8),
                dict(qw=P + 8), dict(kw=P + 2), dict(index=P + 1), dict(seq=P + 2), dict(freqs=P + 4)):
        assert write(lib, c, **bad) == INVALID, bad
    assert write(lib, c, ws=P + 16) == WORKSPACE
    assert write(lib, cache(S=0)) == INVALID
    assert write(lib, c, T=0, q=None, k=None, v=None, index=None, positions=None, out=None) == OK


def test_read_refusals(lib):
    c = cache()
    for bad in (dict(T=-1), dict(T=3), dict(index=None), dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2), dict(index=P + 2), dict(seq=P + 1)):
        assert read(lib, c, **bad) == INVALID, bad
    assert read(lib, c, ws=P + 128) == WORKSPACE
    assert read(lib, c, T=0, index=None, k=None, v=None) == OK


def test_attend_refusals(lib):
    c = cache()
    for bad in (dict(Q=0), dict(Hq=0), dict(Hq=30), dict(Hq=4), dict(scale=float("nan")), dict(scale=float("inf")), dict(node=P, N=-1), dict(node=P, parent=P, N=5, parent_ld=4),
                dict(q=None), dict(lens=None), dict(out=None), dict(q_ld=4088), dict(q_ld=4100), dict(q=P + 8), dict(out=P + 2), dict(lens=P + 2), dict(node=P + 2, N=4),
                dict(node=P, parent=P + 1, N=4, parent_ld=4), dict(lse=P + 2)):
        assert attend(lib, c, **bad) == INVALID, bad
    for bad in (dict(Q=65), dict(Hq=2048, q_ld=2048 * 128), dict(node=P, N=2049)):
        assert attend(lib, c, **bad) == UNSUPPORTED, bad
    assert attend(lib, cache(S=2 ** 31 - 1), Q=2) == UNSUPPORTED
    need = vt.workspace_bytes(vt.VT_OP_KV_ATTEND, n=2, B=1, K=32, V=8, d=128)
    for bad in (dict(ws=None), dict(ws=P + 16), dict(ws_bytes=need - 1), dict(ws_bytes=0)):
        assert attend(lib, c, **bad) == WORKSPACE, bad
    assert attend(lib, cache(S=0), q=None, lens=None, out=None) == OK


def test_commit_refusals(lib):
    c = cache()
    for bad in (dict(N=0), dict(lens=None), dict(path=None), dict(n_accept=None), dict(lens=P + 2), dict(path=P + 1), dict(n_accept=P + 2), dict(nodes=P + 2), dict(new_lens=P + 2)):
        assert commit(lib, c, **bad) == INVALID, bad
    assert commit(lib, c, ws=P + 8) == WORKSPACE
    assert commit(lib, cache(S=0), lens=None, path=None, n_accept=None) == OK


def test_frequency_refusals(lib):
    room = (c_int64 * 128)()
    good = (64, 10000.0, 8.0, 1.0, 4.0, 8192.0)
    assert lib.vt_rope_freqs(*good, room) == OK and lib.vt_rope_freqs(16, 10000.0, 1.0, 0.0, 0.0, 0.0, room) == OK
    nan, inf = float("nan"), float("inf")
    for i, values in ((0, (0, 8, 24, 272, -16)), (1, (1.0, 0.5, nan, inf)), (2, (0.5, nan, inf)), (3, (0.0, -1.0, 4.0, nan)), (4, (1.0, inf, nan)), (5, (0.0, -5.0, nan, inf))):
        for v in values:
            assert lib.vt_rope_freqs(*(v if j == i else g for j, g in enumerate(good)), room) == INVALID, (i, v)
    assert lib.vt_rope_freqs(*good, None) == INVALID
    with pytest.raises(vt.VocabTrimError):
        vt.vt_rope_freqs(24, device="cpu")
    assert vt.vt_rope_freqs(64, device="cpu").shape == (32,)


# ---- the binding ----------------------------------------------------------------------------------------------
class Space:
    ptr, nbytes = 4096, 1 << 30


@pytest.fixture
def calls():
    """The binding bound to functions that record their calls; the library's own again afterwards."""
    real, made, keep = vt.lib(), [], []

    def recorder(name):
        def record(*args):
            made.append((name, args))
            return 0
        keep.append(ctypes.CFUNCTYPE(ctypes.c_int, *getattr(real, name).argtypes)(record))
        return ctypes.cast(keep[-1], c_void_p).value

    vt._bind.use({name: recorder(name) for name in vt._BOUND}, lambda *a: Space(), lambda device: 77, lambda: 0)
    with FakeTensorMode():
        yield made
    vt._lib = None
    vt.lib()


def t(shape, dtype=BF16, device="cuda"):
    return torch.empty(shape, dtype=dtype, device=device)


def args(name, e4m3=False):
    c = (t((9, 8, 16, 128), E4M3 if e4m3 else BF16), t((9, 8, 16, 128), E4M3 if e4m3 else BF16)) + ((t((9, 8, 16), U8), t((9, 8, 16), U8)) if e4m3 else (None, None))
    a = dict(cache=c, pages=t((2, 4), I32))
    if name == "write":
        a.update(q=t((6, 32, 128)), k=t((6, 8, 128)), v=t((6, 8, 128)), index=t(6, I32), seq=t(6, I32), positions=t(6, I32), freqs=t(64, I64), q_weight=t(128),
                 k_weight=t(128), out=t((6, 32, 128)))
    elif name == "read":
        a.update(index=t(6, I32), seq=t(6, I32), out=(t((6, 8, 128)), t((6, 8, 128))))
    elif name == "attend":
        a.update(q=t((6, 32, 128)), lens=t(2, I32), node=t(6, I32), parent=t((2, 20), I32), out=(t((6, 32, 128)), t((6, 32), F32)), ws=Space())
    else:
        a.update(lens=t(2, I32), path=t((2, 7), I32), n_accept=t(2, I32), nodes=t((2, 7), I32), out=t(2, I32))
    return a


CALLS = {"write": vt.vt_qkv_write, "read": vt.vt_kv_read, "attend": vt.vt_kv_attend, "commit": vt.vt_kv_commit}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_call_goes_through_once_on_the_current_stream(calls, name, e4m3):
    CALLS[name](**args(name, e4m3))
    assert len(calls) == 1 and calls[0][1][-1] == 77
    some = args(name, e4m3)
    for optional in ("seq", "out", "q_weight", "nodes", "node"):
        if optional in some:
            some.pop(optional)
            if optional == "node":
                some.pop("parent")
    CALLS[name](**some)
    assert len(calls) == 2


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_kind_are_refused(calls, name):
    for key, value in args(name).items():
        if not isinstance(value, torch.Tensor):
            continue
        for wrong in (t(value.shape, value.dtype, "cpu"), t(value.shape, torch.float64), t((value.shape[0] + 1,) + tuple(value.shape[1:]), value.dtype),
                      t(tuple(value.shape) + (2,), value.dtype)[..., 0], t(value.shape, value.dtype, "cuda:1")):
            if key == "pages" and name in ("write", "read") and wrong.shape[0] != value.shape[0]:
                continue                                            # (with seq, any number of sequences does)
            if wrong.shape == value.shape and wrong.dtype == value.dtype and wrong.is_contiguous() and wrong.device == value.device:
                continue
            with pytest.raises((TypeError, ValueError)):
                CALLS[name](**{**args(name), key: wrong})
    assert not calls


@pytest.mark.parametrize("name", CALLS)
def test_caches_of_another_kind_are_refused(calls, name):
    k, v = args(name)["cache"][:2]
    k8, v8, ke, ve = args(name, True)["cache"]
    for wrong in ((k,), (k, v, None), (k, v8), (k8, v8), (k8, v8, ke, None), (k8, v8, ke, t((9, 8, 15), U8)), (k8, v8, ke, t((9, 8, 16), I32)), (k, v, ke, ve),
                  (k.float(), v.float()), (k[0], v[0]), (k, v[:8]), (k.transpose(2, 3), v.transpose(2, 3)), (k, v.transpose(1, 2).contiguous().transpose(1, 2)),
                  (k, t(k.shape, BF16, "cpu")), (t(k.shape, BF16, "cpu"), v), 5, None):
        with pytest.raises((TypeError, ValueError, AttributeError)):
            CALLS[name](**{**args(name), "cache": wrong})
    assert not calls


def test_shapes_that_do_not_fit_are_refused(calls):
    for bad in (dict(k=t((6, 4, 128))), dict(q=t((5, 32, 128))), dict(q=t((6, 32, 64))), dict(k=t((6, 8, 256))[..., ::2]), dict(v=t((6, 16, 128))[:, ::2]), dict(freqs=t(68, I64)),
                dict(freqs=t(7, I64)), dict(positions=None), dict(q_weight=t(64)), dict(seq=None, pages=t((4, 4), I32)), dict(out=t((6, 32, 64)))):
        with pytest.raises(ValueError):
            vt.vt_qkv_write(**{**args("write"), **bad})
    for bad in (dict(q=t((5, 32, 128))), dict(q=t((6, 30, 128))), dict(q=t((0, 32, 128)), node=None, parent=None), dict(node=None), dict(parent=t((3, 20), I32)),
                dict(parent=t((2, 20, 1), I32)), dict(out=(t((6, 32, 128)), t((6, 31), F32))), dict(lens=t(3, I32)), dict(pages=t((2, 8), I32)[:, ::2])):
        with pytest.raises((ValueError, TypeError)):
            vt.vt_kv_attend(**{**args("attend"), **bad})
    with pytest.raises(ValueError):
        vt.vt_kv_read(args("read")["cache"], t((4, 4), I32), t(6, I32))
    for bad in (dict(path=t((3, 7), I32)), dict(path=t((2, 14), I32)[:, ::2]), dict(nodes=t((2, 6), I32))):
        with pytest.raises(ValueError):
            vt.vt_kv_commit(**{**args("commit"), **bad})
    assert not calls


def test_strides_reach_the_library(calls):
    k = t((9, 16, 8, 128)).transpose(1, 2)
    seen = {}

    def look(*a):
        c = ctypes.cast(a[4], ctypes.POINTER(KV)).contents
        seen.update(page=c.stride_page, head=c.stride_head, token=c.stride_token, heads=c.heads, size=c.page, d=c.d, n=c.n_pages, S=c.S, ld=c.pages_ld, wide=c.max_pages, q_ld=a[1])
        return 0

    real = vt.lib().vt_kv_attend.argtypes
    hold = ctypes.CFUNCTYPE(ctypes.c_int, *real)(look)
    table = {name: 1 for name in vt._BOUND}
    table["vt_kv_attend"] = ctypes.cast(hold, c_void_p).value
    vt._bind.use(table, lambda *a: Space(), lambda device: 77, lambda: 0)
    vt.vt_kv_attend(t((2, 48 * 128)).view(2, 48, 128)[:, 8:40], (k, k), t((2, 6), I32)[:, 1:4], t(2, I32), ws=Space())
    assert seen == dict(page=16 * 8 * 128, head=128, token=8 * 128, heads=8, size=16, d=128, n=9, S=2, ld=6, wide=3, q_ld=48 * 128)
