"""The calls around a tree of drafted tokens without a GPU: arguments that the C calls refuse before any launch, the
binding's own checks, and the oracle's pins."""
import ctypes
import os

import numpy as np
import pytest

from oracle import kv_oracle as K
from oracle import tree_oracle as T
from paper_2606_26650_gb300 import catq as C

OK, ARG, SHAPE, DTYPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 9


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(C.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return C.lib()


def cache(k=1024, v=2048, ks=64, vs=128, table=256, n_pages=10, nkv=2, page=64, d=128, max_pages=4, reserved=0):
    return C.catq_kv_cache(k, v, ks, vs, table, n_pages, nkv, page, d, max_pages, reserved)


def masks(lib, **kw):
    a = dict(parent=64, rs=128, sl=256, B=2, T=8, seen=512, words=1, pos=1024)
    a.update(kw)
    return lib.catq_tree_masks(a["parent"], a["rs"], a["sl"], a["B"], a["T"], a["seen"], a["words"], a["pos"], None)


@pytest.mark.parametrize("want,kw", [
    (OK, dict(T=0)), (OK, dict(B=0)), (SHAPE, dict(T=-1)), (SHAPE, dict(T=1 << 31)), (SHAPE, dict(B=-1)),
    (SHAPE, dict(B=65536)), (SHAPE, dict(words=0)), (SHAPE, dict(words=9)), (ARG, dict(parent=None)), (ARG, dict(rs=None)),
    (ARG, dict(sl=None)), (ARG, dict(seen=None)), (ALIGN, dict(parent=65)), (ALIGN, dict(rs=130)), (ALIGN, dict(sl=257)),
    (ALIGN, dict(seen=514)), (ALIGN, dict(pos=1026)),
])
def test_masks_refuse(lib, want, kw):
    assert masks(lib, **kw) == want


def attend(lib, **kw):
    a = dict(c=cache(), rs=512, sl=640, B=2, seen=128, words=2, Q=4096, ldq=512, T=8, nh=4, O=8192, ldo=512, lse=None,
             ws=65536, n=1 << 40)
    a.update(kw)
    return lib.catq_kv_tree_attention(ctypes.byref(a["c"]), a["rs"], a["sl"], a["B"], a["seen"], a["words"], a["Q"], a["ldq"],
                                      a["T"], a["nh"], a["O"], a["ldo"], a["lse"], a["ws"], a["n"], None)


@pytest.mark.parametrize("want,kw", [
    (OK, dict(T=0)), (OK, dict(B=0)), (OK, dict(T=0, seen=None)), (SHAPE, dict(words=0)), (SHAPE, dict(words=9)),
    (ARG, dict(seen=None)), (ALIGN, dict(seen=130)), (SHAPE, dict(c=cache(d=96))), (SHAPE, dict(nh=3)),
    (SHAPE, dict(ldq=504)), (ARG, dict(Q=None)), (ARG, dict(O=4096, ldo=520)), (ALIGN, dict(O=8194)),
    (ALIGN, dict(lse=66)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(n=1)), (ALIGN, dict(ws=65664)),
])
def test_tree_attention_refuses(lib, want, kw):
    assert attend(lib, **kw) == want


def sample(lib, **kw):
    a = dict(x=4096, ld=1000, dtype=1, R=4, V=1000, t=64, k=128, p=192, m=256, u=320, tokens=384, lp=512)
    a.update(kw)
    return lib.catq_sample(a["x"], a["ld"], a["dtype"], a["R"], a["V"], a["t"], a["k"], a["p"], a["m"], a["u"], a["tokens"],
                           a["lp"], None)


@pytest.mark.parametrize("want,kw", [
    (OK, dict(R=0)), (DTYPE, dict(dtype=2)), (SHAPE, dict(R=-1)), (SHAPE, dict(R=1 << 31)), (SHAPE, dict(V=0)),
    (SHAPE, dict(V=(1 << 20) + 1, ld=1 << 21)), (SHAPE, dict(ld=999)), (ARG, dict(x=None)), (ARG, dict(u=None)),
    (ARG, dict(tokens=None)), (ALIGN, dict(x=4097)), (ALIGN, dict(x=4098, dtype=0)), (ALIGN, dict(t=65)),
    (ALIGN, dict(k=129)), (ALIGN, dict(p=194)), (ALIGN, dict(m=257)), (ALIGN, dict(u=322)), (ALIGN, dict(tokens=385)),
    (ALIGN, dict(lp=514)),
])
def test_sample_refuses(lib, want, kw):
    assert sample(lib, **kw) == want


def accept(lib, **kw):
    a = dict(d=64, s=128, p=192, rs=256, sl=320, B=2, T=8, path=384, kept=448, next=512, len=576)
    a.update(kw)
    return lib.catq_tree_accept(a["d"], a["s"], a["p"], a["rs"], a["sl"], a["B"], a["T"], a["path"], a["kept"], a["next"],
                                a["len"], None)


@pytest.mark.parametrize("want,kw", [
    (OK, dict(B=0)), (SHAPE, dict(B=-1)), (SHAPE, dict(B=65536)), (SHAPE, dict(T=-1)), (SHAPE, dict(T=1 << 31)),
    *[(ARG, {n: None}) for n in ("d", "s", "p", "rs", "sl", "path", "kept", "next", "len")],
    *[(ALIGN, {n: 1025}) for n in ("d", "s", "p", "rs", "sl", "path", "kept", "next", "len")],
])
def test_accept_refuses(lib, want, kw):
    assert accept(lib, **kw) == want


def compact(lib, caches=None, count=None, **kw):
    caches = caches or [cache(), cache()]
    arr = (C.catq_kv_cache * len(caches))(*caches)
    a = dict(rs=512, sl=640, B=2, path=768, kept=896, T=8)
    a.update(kw)
    return lib.catq_kv_compact(arr, len(caches) if count is None else count, a["rs"], a["sl"], a["B"], a["path"], a["kept"],
                               a["T"], None)


@pytest.mark.parametrize("want,kw", [
    (OK, dict(T=0)), (OK, dict(B=0)), (ARG, dict(count=0)), (ARG, dict(count=-1)), (ARG, dict(count=65)),
    (SHAPE, dict(B=-1)), (SHAPE, dict(B=65536)), (SHAPE, dict(T=-1)), (ARG, dict(rs=None)), (ARG, dict(sl=None)),
    (ARG, dict(path=None)), (ARG, dict(kept=None)), (ALIGN, dict(path=770)), (ALIGN, dict(kept=897)), (ALIGN, dict(rs=514)),
    (SHAPE, dict(caches=[cache(), cache(n_pages=11)])), (SHAPE, dict(caches=[cache(), cache(nkv=1)])),
    (SHAPE, dict(caches=[cache(), cache(page=32)])), (SHAPE, dict(caches=[cache(), cache(d=64)])),
    (SHAPE, dict(caches=[cache(), cache(max_pages=5)])), (ARG, dict(caches=[cache(), cache(k=None)])),
    (ALIGN, dict(caches=[cache(), cache(v=2048 + 16)])), (SHAPE, dict(caches=[cache(page=8)])),
    (ARG, dict(caches=[cache(), cache(reserved=1)])),
])
def test_compact_refuses(lib, want, kw):
    assert compact(lib, **kw) == want


def test_compact_takes_no_null_array(lib):
    assert lib.catq_kv_compact(None, 1, 512, 640, 2, 768, 896, 8, None) == ARG
    assert C.catq_kv_compact_max_caches() == 64


def test_the_binding_refuses(lib):
    """Host tensors, wrong dtypes, shapes and sizes raise before the C call."""
    torch = pytest.importorskip("torch")

    def i(*shape):
        return torch.zeros(*shape, dtype=torch.int32)

    with pytest.raises(ValueError):  # host tensors
        C.catq_tree_masks(i(4), i(2), i(1), i(4, 1))
    with pytest.raises(ValueError):
        C.catq_tree_masks(i(4), i(2), i(1), i(3, 1))
    with pytest.raises(ValueError):
        C.catq_tree_masks(i(4), i(2), i(1), i(4))
    with pytest.raises(ValueError):
        C.catq_sample(torch.zeros(4, 10), torch.zeros(4), i(4))
    with pytest.raises(ValueError):
        C.catq_sample(torch.zeros(10), torch.zeros(4), i(4))
    with pytest.raises(ValueError):
        C.catq_tree_accept(i(4), i(4), i(4), i(2), i(1), i(4), i(1), i(1), i(1))
    with pytest.raises(ValueError):
        C.catq_kv_compact([], i(1), i(0), i(0), i(0))


# ------------------------------------------------------------------ the oracle's pins

def test_masks_of_a_small_tree():
    # 0 - 1 - 3, 0 - 2, and a second root 4 with a child
    seen, pos = T.masks([-1, 0, 0, 1, -1, 4], [0, 6], [106], 1)
    assert seen[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b110000]
    assert pos.tolist() == [100, 101, 101, 102, 100, 101]


def test_a_tree_that_is_a_chain_attends_like_single_rows():
    r = np.random.default_rng(0)
    codes = [K.e4m3_encode(np.clip(r.standard_normal((3, 1, 16, 64)) * 50, -448, 448)) for _ in range(2)]
    scale = [np.full((3, 1), 2.0 ** -6) for _ in range(2)]
    q = r.standard_normal((5, 2, 64))
    rs, table = [0, 5], [[2, 0, 1]]
    seen, _ = T.masks([-1, 0, 1, 2, 3], rs, [37], 1)
    a = T.attention(*codes, *scale, table, 16, rs, [37], seen, q, 2)
    b = K.attention(*codes, *scale, table, 16, rs, [37], q, 5, 2)
    for x, y in zip(a, b):
        assert np.allclose(x, y, rtol=1e-12)


def test_sampling_by_hand():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.2, 0.1]))  # in order: 1, 2, 3, 0, 4
    for u, token in ((0.0, 1), (0.39, 1), (0.41, 2), (0.59, 2), (0.61, 3), (0.81, 0), (0.95, 4), (1.0, 4)):
        assert T.sample(x, u)[0] == token, u
    assert abs(T.sample(x, 0.5)[1] - np.log(0.2)) < 1e-9
    assert T.sample(x, 0.99, top_k=2)[0] == 2 and T.sample(x, 0.99, top_k=3)[0] == 3
    assert T.sample(x, 0.99, top_p=0.3)[0] == 1 and T.sample(x, 0.99, top_p=0.45)[0] == 2
    assert T.sample(x, 0.99, top_p=0.0)[0] == 1
    assert T.sample(x, 0.99, min_p=0.4)[0] == 3 and T.sample(x, 0.99, min_p=0.6)[0] == 1 and T.sample(x, 0.99, min_p=9)[0] == 1
    assert T.sample(x, 0.99, temperature=0)[0] == 1
    assert abs(T.sample(x, 0.5, top_k=3, top_p=0.7)[1] - np.log(0.4 / 0.6)) < 1e-9  # 0.7 of 0.8: the first two
    assert T.sample([0.0, 0.0, 0.0], 0.5)[0] == 1 and T.sample([1.0, np.nan], 0.5)[0] == -1
    assert T.sample([-np.inf, 2.0], 0.99)[0] == 1 and T.sample([-np.inf, -np.inf], 0.5)[0] == -1


def test_acceptance_by_hand():
    parent = [-1, 0, 0, 1, 2, 4, -1]
    drafted = [9, 5, 7, 6, 8, 1, 3]
    sampled = [7, 0, 8, 0, 2, 0, 0]  # row 0 draws 7 (row 2), row 2 draws 8 (row 4), row 4 draws 2 (no child)
    path, kept, nxt, new_len = T.accept(drafted, sampled, parent, [0, 7, 7], [50, 3])
    assert path.tolist() == [0, 2, 4, -1, -1, -1, -1] and kept.tolist() == [3, 0]
    assert nxt.tolist() == [2, -1] and new_len.tolist() == [46, 3]


def test_compaction_by_hand():
    # pages of 16: context 14, rows 0 .. 5 at 14 .. 19; kept 0, 3, 5 -> 14, 15, 16
    r = np.random.default_rng(1)
    codes = r.integers(0, 100, (2, 1, 16, 64)).astype(np.uint8)
    scale = np.array([[2.0 ** -4], [2.0 ** 5]])
    before, old = codes.copy(), scale.copy()
    T.compact(codes, scale, [[0, 1]], 16, [0, 6], [20], [0, 3, 5, -1, -1, -1], [3])
    assert scale[1, 0] == old[1, 0] and (codes[1, 0, 0] == before[1, 0, 3]).all()       # row 5: inside its page
    moved = K.E4M3[before[1, 0, 1]] * old[1, 0]                                       # row 3: from 17 to 15
    assert scale[0, 0] == max(old[0, 0], K.scale_of(np.abs(moved).max())) > old[0, 0]
    assert np.allclose(K.E4M3[codes[0, 0, 15]] * scale[0, 0], moved, rtol=2 ** -4, atol=scale[0, 0] * 2 ** -10)
    assert np.allclose(K.E4M3[codes[0, 0, 14]] * scale[0, 0], K.E4M3[before[0, 0, 14]] * old[0, 0], atol=scale[0, 0] * 2 ** -10)
