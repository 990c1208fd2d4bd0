"""GPU parity of the calls around a tree of drafted tokens with the oracle: what the rows see (catq_tree_masks), attention
over the paged 8-bit cache (catq_kv_tree_attention), the accepted branch (catq_tree_accept), its compaction
(catq_kv_compact), and all of them together with drawing tokens.

Tolerances: integers, codes and scales are the oracle's, bit for bit (moved values and scales are exact products of powers of
two, and roundings to e4m3 are to nearest, ties to even, on both sides); attention as in test_gpu_kv.py (the same
arithmetic: half a step of bf16 2^-8 |o|, the three-term weights and fp32 sums (2^-8 + 2^-14) sum p |v|, the weights' floor
2^-17 of the largest)."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from oracle import tree_oracle as O
from paper_2606_26650_gb300 import synthetic as syn
from tests import gpu_util as U
from tests.test_gpu_kv import Paged, bf16, i32, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def device():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def tree(r, n, back=8, roots=1):
    """Parents of n rows: the first `roots` have none, the others one of the `back` before them."""
    return [-1 if i < roots else int(r.integers(max(0, i - back), i)) for i in range(n)]


def trees(r, news, **kw):
    return np.array([p for n in news for p in tree(r, n, **kw)], np.int64)


def done():
    import torch

    from paper_2606_26650_gb300 import catq as C
    torch.cuda.synchronize()
    return C.catq_device_status()


# ------------------------------------------------------------------ what the rows see

@pytest.mark.parametrize("news,words", [
    ([1], 1), ([32], 1), ([5, 0, 31, 7], 1), ([33], 2), ([64, 1], 2), ([65, 96], 3), ([127, 128, 3], 4), ([130], 5),
    ([192], 6), ([200], 7), ([256, 255, 0, 1], 8), ([3, 2], 8), ([3] * 300, 1),
])
@pytest.mark.parametrize("back,roots", [(1, 1), (3, 1), (8, 4), (1000, 2)])
def test_masks_match_oracle(device, news, words, back, roots):
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(40, f"masks/{news[:8]}/{words}/{back}")
    parent, rs = trees(r, news, back=back, roots=roots), starts(news)
    lens = [n + int(r.integers(0, 1000)) for n in news]
    lens[0] = max(news[0] - 1, 0)  # a first position below 0
    T = len(parent)
    seen = torch.full((T + 1, words), 77, dtype=torch.int32, device=device)
    pos = torch.full((T + 1,), 77, dtype=torch.int32, device=device)
    C.catq_tree_masks(i32(parent, device), i32(rs, device), i32(lens, device), seen[:T], pos[:T])
    assert done() == 0
    want, where = O.masks(parent, rs, lens, words)
    assert np.array_equal(seen[:T].cpu().numpy().view(np.uint32), want)
    assert np.array_equal(pos[:T].cpu().numpy(), where)
    assert (seen[T] == 77).all() and pos[T] == 77
    C.catq_tree_masks(i32(parent, device), i32(rs, device), i32(lens, device), seen[:T])  # without positions
    assert done() == 0


def test_masks_of_bad_trees(device):
    """Parents that are not before their rows count as none, sequences out of range are skipped: both latched."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    parent = [-1, 1, 0, 9, -5, 0, 1]

    def run(rs, sl, words=1):
        seen = torch.full((7, words), 77, dtype=torch.int32, device=device)
        C.catq_tree_masks(i32(parent, device), i32(rs, device), i32(sl, device), seen)
        return done(), seen.cpu().numpy()

    status, seen = run([0, 5, 7], [10, 10])
    assert status == 10 and seen[:, 0].tolist() == [1, 2, 5, 8, 16, 1, 2]
    parent = [-1, 0, 1, 2, 3, -1, 0]
    for rs, sl in (([0, 8], [10]), ([-1, 5], [10]), ([5, 0], [10]), ([0, 5], [-1])):
        status, seen = run(rs, sl)
        assert status == 10 and (seen == 77).all()
    parent = list(range(-1, 39))
    seen = torch.full((40, 1), 77, dtype=torch.int32, device=device)
    C.catq_tree_masks(i32(parent, device), i32([0, 33, 40], device), i32([50, 50], device), seen)  # 33 rows, 32 bits
    assert done() == 10 and (seen[:33] == 77).all() and not (seen[33:] == 77).any()


# ------------------------------------------------------------------ attention

def attend(paged, row_start, seq_len, seen, q, nh, device, workspace=None, gap=0):
    import torch

    from paper_2606_26650_gb300 import catq as C
    T, w = q.shape[0], nh * paged.d
    Q = torch.full((T, w + gap), 3.0, dtype=torch.bfloat16, device=device)[:, :w]
    Q.copy_(bf16(q.reshape(T, w), device))
    out = torch.full((T, w + gap), 7.0, dtype=torch.bfloat16, device=device)[:, :w]
    lse = torch.full((T, nh), 7.0, dtype=torch.float32, device=device)
    ws = workspace if workspace is not None else C.kv_attention_workspace(paged.cache, nh)
    bits = torch.from_numpy(np.ascontiguousarray(seen).view(np.int32)).to(device)
    C.catq_kv_tree_attention(paged.cache, i32(row_start, device), i32(seq_len, device), bits, Q, out, nh, ws, lse=lse)
    status = done()
    assert not ws[:4096].any()
    return out.float().cpu().numpy().reshape(T, nh, paged.d).astype(np.float64), lse.cpu().numpy(), status


def check(paged, row_start, seq_len, seen, q, nh, got, lse):
    want, want_lse, mag, low = O.attention(*paged.codes, *paged.scale, paged.table, paged.page, row_start, seq_len, seen,
                                           syn.round_bf16(np.asarray(q, np.float32)), nh)
    outside = np.isnan(want_lse)
    assert (got[outside] == 7).all() and (lse[outside] == 7).all()
    bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -14) * mag + 2.0 ** -17 * low
    off = (np.abs(got - want) - bound)[~outside]
    assert (off <= 0).all(), f"largest excess {off.max():.3g}"
    a, w = lse[~outside], want_lse[~outside]
    seen_any = np.isfinite(w)
    assert (a[~seen_any] == w[~seen_any]).all()
    assert (np.abs(a[seen_any] - w[seen_any]) <= 2.0 ** -16 * (1 + np.abs(w[seen_any]))).all()


@pytest.mark.parametrize("d,nh,nkv,page,lens,news", [
    (128, 2, 2, 64, [1], [1]),                        # one row, no context
    (128, 8, 8, 64, [140], [8]),
    (128, 4, 1, 16, [130, 30], [2, 2]),               # 8 rows a tile
    (128, 8, 2, 64, [200, 129], [4, 3]),              # 16 rows
    (128, 4, 4, 32, [31, 300], [31, 25]),             # 32 rows, a tree with no context, one across tiles
    (128, 12, 4, 128, [257, 120], [16, 13]),          # 64 rows: two row tiles
    (128, 8, 2, 64, [300, 280, 60], [33, 40, 60]),    # 128 rows a tile, two words
    (128, 8, 1, 16, [150, 700], [100, 127]),          # several row tiles of 128, four words
    (128, 4, 1, 64, [400], [256]),                    # as many rows as there are bits
    (64, 6, 2, 16, [77, 260], [5, 20]),
    (64, 4, 4, 32, [513, 255, 256], [7, 1, 3]),
    (64, 8, 1, 64, [600, 90], [64, 90]),
    (64, 3, 3, 128, [300], [256]),
    (64, 2, 1, 16, [9, 40], [3, 4]),
    (128, 4, 1, 64, [9000], [30]),                    # one row tile in as many parts as there are CTAs
    (128, 4, 2, 16, [2500, 1400], [70, 33]),          # parts of several row tiles, an odd number of them
    (64, 4, 1, 128, [8000, 50], [33, 40]),
    (64, 4, 2, 16, [2500, 1400], [70, 33]),
])
@pytest.mark.parametrize("kind", ["tree", "any"])
def test_attention_matches_oracle(device, d, nh, nkv, page, lens, news, kind):
    """kind: a tree's bits; or any, of rows behind too, of some none at all, set beyond the rows."""
    r = syn.rng(41, f"tree/{d}/{nh}/{nkv}/{page}/{lens}/{news}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs = starts(news)
    words = (max(news) + 31) // 32
    if kind == "tree":
        seen, _ = O.masks(trees(r, news), rs, lens, words)
    else:
        seen = r.integers(0, 1 << 32, (rs[-1], words), dtype=np.uint64).astype(np.uint32)
        seen[::3] &= r.integers(0, 1 << 32, seen[::3].shape, dtype=np.uint64).astype(np.uint32)
        seen[::5] = 0
    q = r.standard_normal((rs[-1], nh, d)) * 2.0
    got, lse, status = attend(paged, rs, lens, seen, q, nh, device)
    assert status == 0
    check(paged, rs, np.array(lens), seen, q, nh, got, lse)


def test_a_chain_is_causal_attention(device):
    """Bits up to the row's own give what catq_kv_attention gives, bit for bit: the runs are cut alike."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(42, "chain")
    lens, news, nh = [400, 1000, 70], [24, 24, 24], 8
    paged = Paged(r, lens, 2, 64, 128, device)
    rs = starts(news)
    seen, _ = O.masks(trees(r, news, back=1), rs, lens, 1)
    q = r.standard_normal((rs[-1], nh, 128))
    got, lse, _ = attend(paged, rs, lens, seen, q, nh, device)
    Q, out = bf16(q.reshape(rs[-1], -1), device), torch.empty(rs[-1], nh * 128, dtype=torch.bfloat16, device=device)
    C.catq_kv_attention(paged.cache, i32(rs, device), i32(lens, device), Q, out, nh, C.kv_attention_workspace(paged.cache, nh))
    assert np.abs(got.reshape(rs[-1], -1) - out.float().cpu().numpy()).max() <= 2.0 ** -7 * np.abs(got).max()


def test_rows_apart_idle_slots_and_what_is_out_of_range(device):
    import torch
    r = syn.rng(43, "idle")
    lens, news, nh, d = [90, 0, 50, 40, 2], [3, 0, 5, 40, 4], 4, 64
    paged = Paged(r, [max(n, 1) for n in lens], 2, 16, d, device)
    rs = starts(news)
    seen, _ = O.masks(trees(r, news), rs, lens, 2)
    q = r.standard_normal((rs[-1] + 3, nh, d))           # three rows behind the last sequence
    seen = np.concatenate([seen, np.full((3, 2), 0xFFFFFFFF, np.uint32)])
    got, lse, status = attend(paged, rs, lens, seen, q, nh, device, gap=24)
    assert status == 0 and (got[-3:] == 7).all() and (lse[-3:] == 7).all()
    inside = slice(0, rs[4])                              # the last sequence is shorter than its rows
    want, want_lse, _, _ = O.attention(*paged.codes, *paged.scale, paged.table, 16, rs, lens, seen,
                                       syn.round_bf16(q.astype(np.float32)), nh)
    assert np.abs(got[inside] - want[inside]).max() <= 2.0 ** -6 * np.abs(want[inside]).max()
    last = slice(rs[4], rs[5])
    assert np.abs(got[last] - want[last]).max() <= 2.0 ** -6 * max(np.abs(want[last]).max(), 1e-9)
    assert (np.isinf(lse[last]) == np.isinf(want_lse[last])).all()
    # one word for 40 rows: that sequence is left as it was
    got, lse, status = attend(paged, rs, lens, seen[:, :1], q, nh, device)
    assert status == 10
    assert (got[rs[3]:rs[4]] == 7).all() and not (got[:rs[3]] == 7).any()


def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(device):
    """A page whose scales are NaN: rows whose branch does not enter it, and rows whose context lies before it, are as ever."""
    r = syn.rng(44, "nan")
    nh, d, page = 2, 128, 16
    lens, news = [36], [6]                                # rows at 30 .. 35: two in page 1, four in page 2
    paged = Paged(r, lens, 1, page, d, device)
    rs = starts(news)
    parent = [-1, 0, 0, 1, 1, 2]                          # rows 0 and 1 see nothing of page 2
    seen, _ = O.masks(parent, rs, lens, 1)
    q = r.standard_normal((6, nh, d))
    want, _, _, _ = O.attention(*paged.codes, *paged.scale, paged.table, page, rs, lens, seen,
                                syn.round_bf16(q.astype(np.float32)), nh)
    paged.cache.v_scale[paged.table[0, 2]] = float("nan")
    got, lse, status = attend(paged, rs, lens, seen, q, nh, device)
    assert status == 0
    assert np.isnan(got[2:]).all() and np.isfinite(got[:2]).all()
    assert np.abs(got[:2] - want[:2]).max() <= 2.0 ** -6 * np.abs(want[:2]).max()


# ------------------------------------------------------------------ the accepted branch

@pytest.mark.parametrize("news", [[1], [8], [32, 33, 0, 64, 65], [500, 1, 2], [3] * 700])
@pytest.mark.parametrize("agree", [0.0, 0.5, 1.0])
def test_accept_matches_oracle(device, news, agree):
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(45, f"accept/{news[:5]}/{agree}")
    rs, parent = starts(news), trees(r, news, back=4)
    T = len(parent)
    sampled = r.integers(0, 5, T)                          # few tokens: siblings with the same one
    sampled[r.random(T) < 0.02] = -1                       # nothing could be drawn
    drafted = r.integers(0, 5, T)
    base = np.repeat(rs[:-1], news)
    follow = (r.random(T) < agree) & (parent >= 0)
    drafted[follow] = sampled[base + np.maximum(parent, 0)][follow]
    drafted[r.random(T) < 0.02] = -1
    lens = np.array([n + int(r.integers(0, 100)) for n in news])
    B = len(news)
    path = torch.full((T + 2,), 77, dtype=torch.int32, device=device)
    kept, nxt, new_len = (torch.full((B,), 77, dtype=torch.int32, device=device) for _ in range(3))
    args = [i32(a, device) for a in (drafted, sampled, parent, rs, lens)]
    C.catq_tree_accept(*args, path[:T], kept, nxt, new_len)
    assert done() == 0
    for got, want in zip((path[:T], kept, nxt, new_len), O.accept(drafted, sampled, parent, rs, lens)):
        assert np.array_equal(got.cpu().numpy(), want)
    assert (path[T:] == 77).all()
    C.catq_tree_accept(*args, path[:T], kept, nxt, args[4])  # new lengths over the old
    assert done() == 0 and torch.equal(args[4], new_len)


def test_accept_of_bad_sequences_and_parents(device):
    import torch

    from paper_2606_26650_gb300 import catq as C
    z = i32([0] * 6, device)
    for rs, sl in (([0, 9], [5]), ([-1, 3], [5]), ([4, 2], [5]), ([0, 3], [-2])):
        path = torch.full((6,), 77, dtype=torch.int32, device=device)
        kept, nxt, new_len = (torch.full((1,), 77, dtype=torch.int32, device=device) for _ in range(3))
        C.catq_tree_accept(z, z, z, i32(rs, device), i32(sl, device), path, kept, nxt, new_len)
        assert done() == 10 and (path == 77).all() and kept.item() == 0 and nxt.item() == -1 and new_len.item() == sl[0]
    # parents that are not before their rows are nobody's children
    path = torch.empty(6, dtype=torch.int32, device=device)
    kept, nxt, new_len = (torch.empty(1, dtype=torch.int32, device=device) for _ in range(3))
    C.catq_tree_accept(z, z, i32([0, 1, 5, 3, 9, 0], device), i32([0, 6], device), i32([6], device), path, kept, nxt, new_len)
    assert done() == 0 and path.tolist() == [0, 5, -1, -1, -1, -1] and kept.item() == 2


# ------------------------------------------------------------------ compaction

def branches(r, news, most, moved=True):
    """(path [T], kept [B]): rising places from 0 on."""
    path, kept = [], []
    for n in news:
        m = 0 if n == 0 else int(r.integers(1, min(n, most) + 1))
        way = sorted([0] + list(1 + r.permutation(n - 1)[:m - 1])) if n else []
        if not moved:
            way = list(range(m))
        path += way + [-1] * (n - len(way))
        kept.append(len(way))
    return np.array(path, np.int64), np.array(kept)


@pytest.mark.parametrize("d,nkv,page,lens,news", [
    (128, 1, 64, [64], [1]),                               # nothing to move
    (128, 2, 64, [70, 30], [9, 8]),                        # across a page's end, inside one
    (64, 3, 16, [33, 50, 7, 20], [20, 17, 7, 0]),          # small pages, a sequence of rows alone, an idle one
    (128, 2, 16, [100, 256], [80, 128]),                   # branches over several pages
    (64, 1, 128, [300, 129], [200, 3]),
    (128, 4, 32, [65] * 40, [13] * 40),
    (64, 2, 64, [6], [9]),                                 # a first position below 0
    (64, 2, 16, [700], [600]),                             # more moved tokens than are kept in mind at once
    (128, 1, 128, [600], [500]),
])
@pytest.mark.parametrize("kind", ["alike", "growing", "shrinking", "still"])
@pytest.mark.parametrize("layers", [1, 3])
def test_compact_matches_oracle(device, d, nkv, page, lens, news, kind, layers):
    """kind: scales of neighbouring pages alike; later pages far larger (pages grow, their codes are rounded again) or far
    smaller (what comes is rounded); branches that are in place already."""
    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(46, f"compact/{d}/{nkv}/{page}/{lens[:4]}/{news[:4]}/{kind}")
    rs = starts(news)
    path, kept = branches(r, news, max(news), moved=kind != "still")
    caches = []
    for l in range(layers):
        p = Paged(r, lens, nkv, page, d, device)
        for b in range(len(lens)):
            for i, pg in enumerate(p.table[b][:-(-lens[b] // page)]):
                step = {"growing": 3.0, "shrinking": -3.0}.get(kind, 0.0)
                for x in p.scale:
                    x[pg] = 2.0 ** np.round(-6 + step * i + r.integers(-1, 2, nkv))
        p.scale[1][p.table[0][0], 0] = 0.0                 # a page of zeros takes what comes as it comes
        p.codes[1][p.table[0][0], 0] = 0
        import torch
        for t, x in zip((p.cache.k_scale, p.cache.v_scale), p.scale):
            t.copy_(torch.tensor(x, dtype=torch.float32))
        for t, x in zip((p.cache.k_codes, p.cache.v_codes), p.codes):
            t.view(torch.uint8).copy_(torch.from_numpy(x))
        caches.append(p)
    C.catq_kv_compact([p.cache for p in caches], i32(rs, device), i32(lens, device), i32(path, device), i32(kept, device))
    assert done() == 0
    for p in caches:
        codes, scale = p.host()
        for x, s, got, got_s in zip(p.codes, p.scale, codes, scale):
            before = x.copy()
            O.compact(x, s, p.table, page, rs, lens, path, kept)
            assert np.array_equal(got_s, s)
            assert np.array_equal(K.E4M3[got], K.E4M3[x]), np.argwhere(K.E4M3[got] != K.E4M3[x])[:5]
            if kind == "still":
                assert np.array_equal(got, before)


def test_compact_of_branches_out_of_range(device):
    """Paths that do not rise, rows that are not the sequence's, lengths and pages out of range: left as they were."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(47, "bad")
    paged = Paged(r, [40, 40], 2, 16, 64, device)
    rs, sl = [0, 6, 12], [40, 40]
    whole = [0, 2, 5, -1, -1, -1]

    def run(path, kept, rs=rs, sl=sl, table=None):
        before, scales = paged.host()
        if table is not None:
            paged.cache.table.copy_(i32(table, device))
        C.catq_kv_compact([paged.cache], i32(rs, device), i32(sl, device), i32(path, device), i32(kept, device))
        status = done()
        after, scales2 = paged.host()
        return status, all(np.array_equal(a, b) for a, b in zip(before + scales, after + scales2))

    still = [0, 1, 2, 3, 4, 5]
    for bad in ([0, 2, 2, 3, 4, 5], [0, 6, 7, 8, 9, 10], [2, 1, 5, -1, -1, -1], [-1, 0, 1, 2, 3, 4], [0, 2, 1 << 30, 4, 5, 5]):
        assert run(bad + still, [3, 6]) == (10, True)
    for kept in ([7, 0], [-1, 0]):
        assert run(whole + still, kept) == (10, True)
    for rs_, sl_ in (([0, 13, 12], sl), ([-1, 6, 12], sl), (rs, [40, 49]), (rs, [-3, 40])):
        assert run(whole + still, [3, 6], rs_, sl_)[0] == 10
    table = paged.table.copy()
    table[0, :] = 1 << 20
    assert run(whole + still, [3, 6], table=table) == (10, True)


def test_compact_of_pages_that_are_not_finite(device):
    """A token from a page whose scale is NaN makes the page that it enters NaN; moves beside it are as ever."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(48, "nan")
    paged = Paged(r, [36, 36], 1, 16, 64, device)
    for x in paged.scale:
        x[:] = 2.0 ** -6
    paged.scale[0][paged.table[0, 2]] = np.nan
    for t, x in zip((paged.cache.k_scale, paged.cache.v_scale), paged.scale):
        t.copy_(torch.tensor(x, dtype=torch.float32))
    rs, sl, path, kept = [0, 6, 12], [36, 36], [0, 4, 5, -1, -1, -1] * 2, [3, 3]  # 30, 31, 32
    C.catq_kv_compact([paged.cache], i32(rs, device), i32(sl, device), i32(path, device), i32(kept, device))
    assert done() == 0
    codes, scale = paged.host()
    for x, s, got, got_s in zip(paged.codes, paged.scale, codes, scale):
        O.compact(x, s, paged.table, 16, rs, sl, path, kept)
        assert np.array_equal(got_s, s, equal_nan=True)
        assert np.array_equal(K.E4M3[got], K.E4M3[x])
    assert np.isnan(scale[0][paged.table[0, 1]]).all() and np.isfinite(scale[0][paged.table[1, 1]]).all()


def test_compact_behind_the_first_4_gb(device):
    """Pages whose codes lie behind 2^32 bytes."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    n_pages, page, d = 300000, 128, 128
    table = i32([[n_pages - 2, n_pages - 1]], device)
    codes = [torch.empty(n_pages, 1, page, d, dtype=torch.uint8, device=device) for _ in range(2)]
    scales = [torch.ones(n_pages, 1, device=device) for _ in range(2)]
    for x in codes:
        x[-2:] = (torch.arange(2 * page, device=device) % 100).to(torch.uint8).view(2, 1, page, 1)
    cache = C.KVCache(*(x.view(torch.float8_e4m3fn) for x in codes), *scales, table)
    C.catq_kv_compact([cache], i32([0, 8], device), i32([132], device), i32([0, 2, 6, 7, -1, -1, -1, -1], device), i32([4], device))
    assert done() == 0
    for x in codes:
        got = x[-2:].view(2 * page, d)
        for slot, token in zip(range(124, 128), (124, 126, 130, 131)):
            assert (got[slot] == token % 100).all()
        assert (got[:124, 0].cpu() == torch.arange(124) % 100).all()


# ------------------------------------------------------------------ together

def test_two_captured_graphs_at_once(device):
    """Two graphs with workspaces of their own, replayed on two streams, give what they give alone."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(51, "graphs")
    graphs, outs, want = [], [], []
    for d, nh, nkv, lens, news in ((128, 8, 1, [3000, 900], [24, 31]), (64, 8, 2, [2000, 100], [40, 7])):
        paged = Paged(r, lens, nkv, 16, d, device)
        rs = starts(news)
        seen, _ = O.masks(trees(r, news), rs, lens, 2)
        T = int(rs[-1])
        q, out = bf16(r.standard_normal((T, nh * d)), device), torch.empty(T, nh * d, dtype=torch.bfloat16, device=device)
        args = (paged.cache, i32(rs, device), i32(lens, device), torch.from_numpy(seen.view(np.int32)).to(device), q, out, nh,
                C.kv_attention_workspace(paged.cache, nh))
        C.catq_kv_tree_attention(*args)
        torch.cuda.synchronize()
        want.append(out.clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            C.catq_kv_tree_attention(*args)
        graphs.append((g, args))
        outs.append(out)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for (g, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        assert done() == 0
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def step_tensors(device, B, T, nh, nkv, d, V, words):
    import torch
    e = dict(device=device)
    return dict(seen=torch.zeros(T, words, dtype=torch.int32, **e), pos=torch.zeros(T, dtype=torch.int32, **e),
                tokens=torch.zeros(T, dtype=torch.int32, **e), path=torch.zeros(T, dtype=torch.int32, **e),
                kept=torch.zeros(B, dtype=torch.int32, **e), next=torch.zeros(B, dtype=torch.int32, **e),
                new_len=torch.zeros(B, dtype=torch.int32, **e), out=torch.zeros(T, nh * d, dtype=torch.bfloat16, **e),
                logits=torch.zeros(T, V, dtype=torch.bfloat16, **e))


@pytest.mark.parametrize("captured", [False, True])
def test_drafted_steps_follow_plain_decoding(device, captured):
    """Greedy decoding of a one-layer model whose logits are the packed projection of the attention's output: steps that
    check a tree, accept and compact go through the same tokens as decoding them one by one, and attention sees the same
    cache, whether the step is launched or replayed as a graph."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(49, "steps")
    nh, nkv, d, page, B, V, g = 4, 2, 64, 16, 2, 256, 64
    wide = nh * d
    W = syn.round_bf16(r.standard_normal((V, wide)).astype(np.float32) * 0.05)
    layer = C.Layer.create(U.to_device(W, "bf16", device), g)
    C.catq_group_stats(layer)
    codes = torch.empty(V * wide // 4, dtype=torch.uint8, device=device)
    alpha = torch.empty(V * wide // g, dtype=torch.float32, device=device)
    C.catq_hard_ternarize_pack(layer, codes, alpha)
    embed = bf16(r.standard_normal((V, wide + 2 * nkv * d)), device)  # a token's query, key and value
    rope = C.Rope.create(d, 10000.0, device)
    prompt = [11, 30]
    parent, N = [-1, 0, 0, 1, 1, 2, 3], 7
    max_pages = 6

    def fresh():
        table = torch.arange(B * max_pages, dtype=torch.int32, device=device).reshape(B, max_pages)
        return C.KVCache.create(B * max_pages, nkv, page, d, table)

    def qkv(tokens):
        x = embed[tokens.long()]
        return x[:, :wide].contiguous(), x[:, wide:wide + nkv * d], x[:, wide + nkv * d:]

    def fill(cache):
        rs, sl = i32(starts(prompt), device), i32(prompt, device)
        q, k, v = qkv(i32(syn.rng(50, "prompt").integers(0, V, sum(prompt)), device))
        C.catq_kv_append(cache, rs, sl, k, v, rope=rope)
        return sl

    # one by one
    def plain(steps):
        cache = fresh()
        ws = C.kv_attention_workspace(cache, nh)
        lens, out = fill(cache), []
        token = i32([3, 5], device)
        rs = i32([0, 1, 2], device)
        logits = torch.empty(B, V, dtype=torch.bfloat16, device=device)
        u = torch.full((B,), 0.5, device=device)
        zero = torch.zeros(B, device=device)
        for _ in range(steps):
            q, k, v = qkv(token)
            lens = lens + 1
            o = torch.empty(B, wide, dtype=torch.bfloat16, device=device)
            C.catq_kv_append(cache, rs, lens, k, v, rope=rope, Q=q, n_heads=nh)
            C.catq_kv_attention(cache, rs, lens, q, o, nh, ws)
            C.catq_ternary_infer(codes, alpha, V, wide, g, o, logits)
            token = torch.empty(B, dtype=torch.int32, device=device)
            C.catq_sample(logits, u, token, temperature=zero)
            out.append(token.cpu().numpy())
        return np.array(out).T

    want = plain(14)
    cache = fresh()
    ws = C.kv_attention_workspace(cache, nh)
    lens = fill(cache)
    T = B * N
    s = step_tensors(device, B, T, nh, nkv, d, V, 1)
    rs, par = i32([0, N, T], device), i32(parent * B, device)
    drafted, sl = torch.zeros(T, dtype=torch.int32, device=device), torch.zeros(B, dtype=torch.int32, device=device)
    u, zero = torch.full((T,), 0.5, device=device), torch.zeros(T, device=device)

    def step():
        x = embed[drafted.long()]
        q, k, v = x[:, :wide], x[:, wide:wide + nkv * d], x[:, wide + nkv * d:]
        C.catq_tree_masks(par, rs, sl, s["seen"], s["pos"])
        C.catq_rope_at(q, s["pos"], rope, nh, d)
        C.catq_rope_at(k, s["pos"], rope, nkv, d)
        C.catq_kv_append(cache, rs, sl, k, v)
        C.catq_kv_tree_attention(cache, rs, sl, s["seen"], q, s["out"], nh, ws)
        C.catq_ternary_infer(codes, alpha, V, wide, g, s["out"], s["logits"])
        C.catq_sample(s["logits"], u, s["tokens"], temperature=zero)
        C.catq_tree_accept(drafted, s["tokens"], par, rs, sl, s["path"], s["kept"], s["next"], s["new_len"])
        C.catq_kv_compact([cache], rs, sl, s["path"], s["kept"])

    graph = None
    if captured:
        saved = [t.clone() for t in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)]
        sl.copy_(lens + N)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for t, x in zip((cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale), saved):
            t.copy_(x)
    token, got, kept_all = np.array([3, 5]), [[], []], []
    for it in range(3):
        rows = r.integers(0, V, T)
        for b in range(B):
            rows[b * N] = token[b]
            upcoming = want[b][len(got[b]):]
            # the branch 0 - 1 - 3 - 6 holds the right tokens, as far as the step lets it
            for at, row in zip(range(1 + (it + b) % 3), (1, 3, 6)):
                rows[b * N + row] = upcoming[at]
        drafted.copy_(i32(rows, device))
        sl.copy_(lens + N)
        if graph is None:
            step()
        else:
            graph.replay()
        assert done() == 0
        kept, path, tokens = s["kept"].cpu().numpy(), s["path"].cpu().numpy().reshape(B, N), s["tokens"].cpu().numpy()
        kept_all.append(kept.tolist())
        for b in range(B):
            got[b] += [int(tokens[b * N + i]) for i in path[b][:kept[b]]]
        lens = s["new_len"].clone()
        token = s["next"].cpu().numpy()
    # bf16 keys are rounded before the code here and not there: a token may differ where two logits are all but equal
    for b in range(B):
        assert got[b] == want[b][:len(got[b])].tolist(), (got[b], want[b])
    assert max(max(k) for k in kept_all) >= 3


# ------------------------------------------------------------------ beside the causal call; rows without a context

def chained(device, d, nh, nkv, page, lens, news, words):
    """(tree's and causal attention of the same rows, the larger of the two parts' sums p |v|)."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(52, f"chain/{d}/{nh}/{nkv}/{lens}/{news}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs = starts(news)
    seen, _ = O.masks(trees(r, news, back=1), rs, lens, words)
    q = r.standard_normal((rs[-1], nh, d)) * 2.0
    got, lse, status = attend(paged, rs, lens, seen, q, nh, device)
    assert status == 0
    out = torch.full((int(rs[-1]), nh * d), 7.0, dtype=torch.bfloat16, device=device)
    lse2 = torch.full((int(rs[-1]), nh), 7.0, device=device)
    C.catq_kv_attention(paged.cache, i32(rs, device), i32(lens, device), bf16(q.reshape(rs[-1], -1), device), out, nh,
                        C.kv_attention_workspace(paged.cache, nh), lse=lse2)
    assert done() == 0
    _, _, mag, low = O.attention(*paged.codes, *paged.scale, paged.table, page, rs, lens, seen,
                                 syn.round_bf16(np.asarray(q, np.float32)), nh)
    return got, lse, out.float().cpu().numpy().reshape(got.shape).astype(np.float64), lse2.cpu().numpy(), mag, low


@pytest.mark.parametrize("d,nh,nkv,page,lens,news,words", [
    (128, 4, 2, 64, [100, 128, 3], [2, 4, 3], 1),          # tiles of 8 rows
    (128, 8, 2, 16, [100, 128, 70], [4, 3, 4], 1),         # of 16
    (128, 8, 2, 64, [100, 128, 70], [8, 8, 7], 1),         # of 32
    (128, 8, 2, 64, [128, 127, 100], [33, 40, 60], 2),     # of 128
    (64, 8, 4, 32, [256, 200, 31], [4, 4, 3], 1),
    (64, 8, 2, 16, [256, 255, 90], [16, 15, 9], 1),
])
def test_chains_of_one_tile_of_tokens_are_causal_attention(device, d, nh, nkv, page, lens, news, words):
    """Where no row tile's tokens are shared out and both calls take tiles of as many rows, they do the same arithmetic: equal
    bits."""
    got, lse, want, want_lse, _, _ = chained(device, d, nh, nkv, page, lens, news, words)
    assert np.array_equal(got, want) and np.array_equal(lse, want_lse)


@pytest.mark.parametrize("d,nh,nkv,page,lens,news,words", [
    (128, 8, 2, 64, [400, 1000, 70], [24, 24, 24], 1),
    (128, 8, 1, 16, [9000, 600], [100, 127], 4),
    (64, 8, 2, 64, [5000, 1000], [30, 17], 1),
])
def test_chains_are_causal_attention(device, d, nh, nkv, page, lens, news, words):
    """Shared out otherwise: two outputs that are each within the oracle's bounds, element by element, and twice the part of these
    that is not the last rounding."""
    got, lse, want, want_lse, mag, low = chained(device, d, nh, nkv, page, lens, news, words)
    bound = 2.0 ** -8 * (np.abs(got) + np.abs(want)) + 2 * ((2.0 ** -8 + 2.0 ** -14) * mag + 2.0 ** -17 * low)
    assert (np.abs(got - want) <= bound).all()
    assert (np.abs(lse - want_lse) <= 2.0 ** -15 * (1 + np.abs(want_lse))).all()


@pytest.mark.parametrize("d,nh,nkv,page,lens,news", [
    (128, 1, 1, 64, [256] + [3] * 40, [256] + [1] * 40),    # 8 rows a tile: two tiles of tokens, the first hidden from many rows
    (128, 2, 1, 16, [256] + [2] * 40, [256] + [2] * 40),    # 16
    (128, 4, 1, 16, [256] + [5] * 40, [256] + [2] * 40),    # 32
    (128, 2, 1, 64, [256, 129], [256, 129]),                # 128
    (64, 2, 1, 16, [256, 200], [256, 200]),
    (64, 2, 2, 32, [256, 140], [250, 140]),
])
@pytest.mark.parametrize("kind", ["alone", "late", "none"])
def test_rows_from_which_whole_tiles_are_hidden(device, d, nh, nkv, page, lens, news, kind):
    """Trees without a context (or of a few tokens): rows that see themselves alone, or rows from the 128th on, or nothing."""
    r = syn.rng(53, f"hidden/{d}/{nh}/{nkv}/{lens[:2]}/{news[:2]}/{kind}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs = starts(news)
    words = 8
    seen = np.zeros((int(rs[-1]), words), np.uint32)
    for b, n in enumerate(news):
        for i in range(n):
            if kind == "alone":
                seen[rs[b] + i, i // 32] = np.uint32(1 << (i % 32))
            elif kind == "late":
                seen[rs[b] + i, 4:] = r.integers(0, 1 << 32, 4, dtype=np.uint64).astype(np.uint32)
    q = r.standard_normal((int(rs[-1]), nh, d)) * 2.0
    got, lse, status = attend(paged, rs, lens, seen, q, nh, device)
    assert status == 0
    check(paged, rs, np.array(lens), seen, q, nh, got, lse)
