"""The decoding calls without a GPU: arguments that the C calls refuse before any launch, the binding's own checks, the
frequencies, and the oracle's pins."""
import ctypes
import os

import numpy as np
import pytest

from oracle import kv_oracle as K
from paper_2606_26650_gb300 import catq as C

OK, ARG, SHAPE, DTYPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(C.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return C.lib()


def rot(turns=64, rot=64, layout=0, magnitude=1.0, reserved=0):
    return ctypes.byref(C.catq_rotation(turns, rot, layout, magnitude, reserved))


def cache(k=1024, v=2048, ks=64, vs=128, table=256, n_pages=10, nkv=2, page=64, d=128, max_pages=4, reserved=0):
    return ctypes.byref(C.catq_kv_cache(k, v, ks, vs, table, n_pages, nkv, page, d, max_pages, reserved))


@pytest.mark.parametrize("want,kw", [
    (OK, dict(T=0)),
    (DTYPE, dict(dtype=2)), (SHAPE, dict(T=-1)), (SHAPE, dict(nh=0)), (SHAPE, dict(d=63)), (SHAPE, dict(ldx=511)),
    (SHAPE, dict(ldy=511)), (SHAPE, dict(r=rot(rot=130))), (SHAPE, dict(r=rot(rot=5))), (SHAPE, dict(r=rot(rot=0))),
    (ARG, dict(r=None)), (ARG, dict(r=rot(turns=0))), (ARG, dict(r=rot(layout=2))), (ARG, dict(r=rot(reserved=1))),
    (ARG, dict(r=rot(magnitude=float("inf")))), (ALIGN, dict(r=rot(turns=68))), (ARG, dict(X=None)), (ARG, dict(Y=None)),
    (ARG, dict(pos=None)), (ARG, dict(Y=4096, ldy=520)), (ALIGN, dict(X=4097)), (ALIGN, dict(dtype=0, X=4098)),
    (ALIGN, dict(pos=66)),
])
def test_rope_at_refuses(lib, want, kw):
    a = dict(X=4096, ldx=512, Y=8192, ldy=512, dtype=1, pos=64, T=8, nh=4, d=128, r=rot())
    a.update(kw)
    got = lib.catq_rope_at(a["X"], a["ldx"], a["Y"], a["ldy"], a["dtype"], a["pos"], a["T"], a["nh"], a["d"], a["r"], 0,
                           None)
    assert got == want


CACHE_ERRORS = [
    (SHAPE, dict(d=96)), (SHAPE, dict(page=8)), (SHAPE, dict(page=48)), (SHAPE, dict(page=256)), (SHAPE, dict(nkv=0)),
    (SHAPE, dict(nkv=4097)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(max_pages=0)), (SHAPE, dict(n_pages=1 << 25, nkv=1)),
    (SHAPE, dict(max_pages=(1 << 24) + 1)), (ARG, dict(reserved=1)), (ARG, dict(k=None)), (ARG, dict(v=None)),
    (ARG, dict(ks=None)), (ARG, dict(vs=None)), (ARG, dict(table=None)), (ALIGN, dict(k=1024 + 64)),
    (ALIGN, dict(v=2048 + 16)), (ALIGN, dict(ks=66)), (ALIGN, dict(vs=65)), (ALIGN, dict(table=258)),
]


def append(lib, **kw):
    a = dict(c=cache(), rs=512, sl=640, B=2, K=4096, ldk=256, V=8192, ldv=256, T=8, Q=16384, ldq=512, Qo=32768, ldqo=512,
             nh=4, r=rot())
    a.update(kw)
    return lib.catq_kv_append(a["c"], a["rs"], a["sl"], a["B"], a["K"], a["ldk"], a["V"], a["ldv"], a["T"], a["Q"],
                              a["ldq"], a["Qo"], a["ldqo"], a["nh"], a["r"], None)


def attend(lib, **kw):
    a = dict(c=cache(), rs=512, sl=640, B=2, Q=4096, ldq=512, T=8, nh=4, O=8192, ldo=512, lse=None, ws=65536, n=1 << 40)
    a.update(kw)
    return lib.catq_kv_attention(a["c"], a["rs"], a["sl"], a["B"], a["Q"], a["ldq"], a["T"], a["nh"], a["O"], a["ldo"],
                                 a["lse"], a["ws"], a["n"], None)


@pytest.mark.parametrize("want,kw", CACHE_ERRORS)
def test_caches_are_checked(lib, want, kw):
    assert append(lib, c=cache(**kw)) == want
    assert attend(lib, c=cache(**kw)) == want


@pytest.mark.parametrize("want,kw", [
    (OK, dict(T=0)), (OK, dict(B=0)), (ARG, dict(c=None)), (SHAPE, dict(B=-1)), (SHAPE, dict(B=65536)), (SHAPE, dict(T=-1)),
    (SHAPE, dict(T=1 << 31)), (ARG, dict(rs=None)), (ARG, dict(sl=None)), (ALIGN, dict(rs=514)), (ALIGN, dict(sl=642)),
])
def test_sequences_are_checked(lib, want, kw):
    assert append(lib, **kw) == want
    assert attend(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (SHAPE, dict(ldk=255)), (SHAPE, dict(ldv=248)), (SHAPE, dict(ldq=504)), (SHAPE, dict(ldqo=504)), (SHAPE, dict(nh=0)),
    (SHAPE, dict(r=rot(rot=24))), (SHAPE, dict(r=rot(rot=144))), (ARG, dict(r=rot(turns=0))), (ARG, dict(K=None)),
    (ARG, dict(V=None)), (ARG, dict(Qo=None)), (ARG, dict(Qo=16384, ldqo=520)), (ALIGN, dict(K=4104)), (ALIGN, dict(V=8200)),
    (ALIGN, dict(ldk=260)), (ALIGN, dict(ldv=258)), (ALIGN, dict(Q=16388)), (ALIGN, dict(ldqo=516)),
])
def test_append_refuses(lib, want, kw):
    assert append(lib, **kw) == want


@pytest.mark.parametrize("want,kw", [
    (SHAPE, dict(nh=3)), (SHAPE, dict(nh=0)), (SHAPE, dict(nh=2 * 65, ldq=1 << 15, ldo=1 << 15)), (SHAPE, dict(ldq=504)),
    (SHAPE, dict(ldo=504)), (SHAPE, dict(T=(1 << 25) + 1)), (ARG, dict(Q=None)), (ARG, dict(O=None)),
    (ARG, dict(O=4096, ldo=520)), (ALIGN, dict(Q=4104)), (ALIGN, dict(O=8194)), (ALIGN, dict(ldq=516)),
    (ALIGN, dict(lse=66)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(n=1)), (ALIGN, dict(ws=65664)),
])
def test_attention_refuses(lib, want, kw):
    assert attend(lib, **kw) == want


def test_workspace_sizes(lib):
    assert lib.catq_kv_attention_workspace_bytes(32, 8, 128) % 256 == 0
    assert lib.catq_kv_attention_workspace_bytes(32, 8, 128) > lib.catq_kv_attention_workspace_bytes(12, 4, 64) > 4096
    assert lib.catq_kv_attention_workspace_bytes(10, 4, 128) == 0
    assert lib.catq_kv_attention_workspace_bytes(8, 4, 96) == 0


@pytest.mark.parametrize("scaling", ["plain", "linear", "bands", "yarn"])
@pytest.mark.parametrize("rot_,base", [(128, 500000.0), (64, 10000.0), (10, 10000.0), (2, 10000.0)])
def test_turns_follow_the_oracle(lib, scaling, rot_, base):
    kw = dict(factor=8.0, low=1.0, high=32.0 if scaling == "yarn" else 4.0, original=8192.0)
    freq, magnitude = K.frequencies(rot_, base, scaling, **kw)
    turns, got = C.catq_rotation_turns(rot_, base, ["plain", "linear", "bands", "yarn"].index(scaling), **kw)
    # fp64 on both sides (a relative 2^-50 for powers and quotients), then 2^-62 of a turn
    want = freq / (2 * np.pi)
    assert np.all(np.abs(np.array(turns, np.float64) * 2.0 ** -64 - want) <= want * 2.0 ** -50 + 2.0 ** -62)
    assert abs(got - magnitude) <= 2.0 ** -23 * magnitude


@pytest.mark.parametrize("want,kw", [
    (SHAPE, dict(rot=7)), (SHAPE, dict(rot=0)), (SHAPE, dict(rot=65538)), (ARG, dict(base=1.0)),
    (ARG, dict(base=float("nan"))), (ARG, dict(scaling=4)), (ARG, dict(scaling=-1)), (ARG, dict(scaling=1, factor=0.5)),
    (ARG, dict(scaling=2, low=0.0)), (ARG, dict(scaling=2, low=4.0, high=4.0)), (ARG, dict(scaling=3, original=0.0)),
    (ARG, dict(scaling=3, high=float("inf"))),
])
def test_turns_refuse(lib, want, kw):
    a = dict(rot=8, base=10000.0, scaling=0, factor=2.0, low=1.0, high=4.0, original=64.0)
    a.update(kw)
    turns, m = (ctypes.c_int64 * 4)(), ctypes.c_float()
    assert lib.catq_rotation_turns(a["rot"], a["base"], a["scaling"], a["factor"], a["low"], a["high"], a["original"],
                                   turns, ctypes.byref(m)) == want
    assert lib.catq_rotation_turns(8, 1e4, 0, 1.0, 1.0, 4.0, 64.0, None, ctypes.byref(m)) == ARG


class Fake:
    """Stands in for a CUDA tensor: what the binding's checks read."""

    def __init__(self, shape, dtype, stride=None, cuda=True):
        import torch
        self.shape, self.dtype, self.is_cuda = tuple(shape), getattr(torch, dtype), cuda
        self._e = torch.empty((), dtype=self.dtype).element_size()
        self._s = stride or tuple(int(np.prod(shape[i + 1:])) for i in range(len(shape)))
        self.device = "cuda"

    def stride(self):
        return self._s

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self._e

    def is_contiguous(self):
        return self._s == tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))

    def data_ptr(self):
        return 4096


def test_binding_refuses_before_the_library():
    pytest.importorskip("torch")
    codes, scale = Fake((6, 2, 16, 64), "uint8"), Fake((6, 2), "float32")
    table = Fake((3, 4), "int32")
    c = C.KVCache(codes, codes, scale, scale, table)
    assert (c.B, c.n_kv_heads, c.page, c.d) == (3, 2, 16, 64) and c.struct().max_pages == 4
    for bad in [(Fake((6, 2, 16, 64), "bfloat16"), codes, scale, scale, table),
                (codes, Fake((5, 2, 16, 64), "uint8"), scale, scale, table),
                (codes, codes, Fake((6, 2), "bfloat16"), scale, table),
                (codes, codes, scale, Fake((5, 2), "float32"), table),
                (codes, codes, scale, scale, Fake((3, 4), "int64")),
                (codes, codes, scale, scale, Fake((3, 4), "int32", cuda=False))]:
        with pytest.raises(ValueError):
            C.KVCache(*bad)
    with pytest.raises(ValueError):
        C.Rope(Fake((31,), "int64"), 64)
    with pytest.raises(ValueError):
        C.Rope(Fake((32,), "int32"), 64)
    rs, sl = Fake((4,), "int32"), Fake((3,), "int32")
    K_, Q = Fake((5, 128), "bfloat16"), Fake((5, 256), "bfloat16")
    for kw in [dict(row_start=Fake((3,), "int32")), dict(seq_len=Fake((2,), "int32")), dict(row_start=Fake((4,), "int64")),
               dict(K=Fake((5, 128), "float32")), dict(K=Fake((5, 64), "bfloat16")), dict(V=Fake((4, 128), "bfloat16")),
               dict(V=Fake((5, 128), "bfloat16", stride=(64, 1))), dict(V=Fake((5, 128), "bfloat16", stride=(256, 2))),
               dict(K=Fake((5, 2, 64), "bfloat16", stride=(256, 128, 1))), dict(K=Fake((5, 128), "bfloat16", cuda=False))]:
        a = dict(row_start=rs, seq_len=sl, K=K_, V=K_)
        a.update(kw)
        with pytest.raises(ValueError):
            C.catq_kv_append(c, **a)
    for kw in [dict(Q=Fake((5, 250), "bfloat16")), dict(O=Fake((5, 256), "float32")), dict(lse=Fake((5, 3), "float32")),
               dict(seq_len=Fake((2,), "int32"))]:
        a = dict(row_start=rs, seq_len=sl, Q=Q, O=Q, n_heads=4, workspace=Fake((64,), "uint8"))
        a.update(kw)
        with pytest.raises(ValueError):
            C.catq_kv_attention(c, **a)
    r = C.Rope(Fake((32,), "int64"), 64)
    with pytest.raises(ValueError):
        C.catq_rope_at(Q, Fake((4,), "int32"), r, 4, 64)
    with pytest.raises(ValueError):
        C.catq_rope_at(Q, Fake((5,), "int32"), r, 4, 64, Y=Fake((5, 256), "float32"))


# ------------------------------------------------------------------ the oracle's pins

def test_oracle_e4m3_numbers():
    assert K.E4M3[0x7E] == 448 and K.E4M3[0x01] == 2.0 ** -9 and K.E4M3[0x38] == 1.0 and np.isnan(K.E4M3[0x7F])
    assert np.array_equal(K.E4M3[K.e4m3_encode(K.E4M3[:127])], K.E4M3[:127])
    # ties go to the even code: 1 + 1/16 lies between 1 (0x38) and 1.125 (0x39), 1.1875 between 0x39 and 0x3A
    assert list(K.e4m3_encode([1 + 1 / 16, 1 + 3 / 16, -1 - 1 / 16, 2.0 ** -10, 3 * 2.0 ** -10, 464.0])) == \
        [0x38, 0x3A, 0xB8, 0x00, 0x02, 0x7E]
    torch = pytest.importorskip("torch")
    x = torch.linspace(-448, 448, 20001, dtype=torch.float32)
    assert np.array_equal(K.e4m3_encode(x.numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_oracle_scales():
    assert K.scale_of(448.0) == 1.0 and K.scale_of(448.0001) == 2.0 and K.scale_of(0.0) == 0.0
    assert K.scale_of(1e-30) == 2.0 ** -60 and np.isnan(K.scale_of(np.inf)) and K.scale_of(1.75) == 2.0 ** -8


def test_oracle_rotation_keeps_lengths_and_turns_back():
    r = np.random.default_rng(0)
    x = r.standard_normal((5, 2, 16))
    freq, _ = K.frequencies(8, 100.0)
    for inter in (False, True):
        y = K.rope(x, np.arange(5) * 7, freq, inter)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 8:], x[..., 8:])
        assert np.allclose(K.rope(y, np.arange(5) * 7, freq, inter, inverse=True), x)
        assert np.allclose(y[0], x[0])


def test_oracle_attention_by_hand():
    """Two tokens, one head: the second query sees both, the first only the first."""
    codes = K.e4m3_encode(np.array([[[[1.0] * 4 + [0.0] * 4, [0.0] * 4 + [2.0] * 4]]]))  # [1 page, 1 head, 2 tokens, 8]
    one = np.ones((1, 1))
    q = np.zeros((2, 1, 8))
    q[1, 0, 4:] = 1.0
    O, lse, _, _ = K.attention(codes, codes, one, one * 2, [[0]], 2, [0, 2], [2], q, 2, 1)
    w = np.exp(8 / np.sqrt(8))
    assert np.allclose(O[0, 0], [2.0] * 4 + [0.0] * 4) and np.allclose(lse[0, 0], 0.0)
    assert np.allclose(O[1, 0], np.array([2.0] * 4 + [4.0 * w] * 4) / (1 + w)) and np.allclose(lse[1, 0], np.log(1 + w))


def test_heads_of_64_take_the_workspace_of_tiles_of_32_rows(lib):
    """The size that the query gives is the tree call's; this call of heads of 64 has no tiles of 128 rows and takes half of
    the parts' bytes.  (A size that is enough is told from one that is not by the refusal that comes next.)"""
    whole = lib.catq_kv_attention_workspace_bytes(4, 2, 64)
    half = 4096 + (whole - 4096) // 2
    off = 65536 + 64

    def call(n):
        return attend(lib, c=cache(d=64), ldq=256, ldo=256, ws=off, n=n)

    assert call(half) == call(whole) == ALIGN and call(half - 256) == WORKSPACE
    c = cache(d=64)
    tree = [lib.catq_kv_tree_attention(c, 512, 640, 2, 128, 1, 4096, 256, 8, 4, 8192, 256, None, off, n, None)
            for n in (whole, whole - 256, half)]
    assert tree == [ALIGN, WORKSPACE, WORKSPACE]
    whole = lib.catq_kv_attention_workspace_bytes(4, 2, 128)  # (heads of 128 have those tiles in either call)
    assert attend(lib, ws=off, n=whole) == ALIGN and attend(lib, ws=off, n=whole - 256) == WORKSPACE
