"""GPU parity of the decoding operators with the fp64 oracle: rotary positions (catq_rope_at), the append to the paged
8-bit cache (catq_kv_append), attention over it (catq_kv_attention), and the three together with the packed linears.

Tolerances, from the arithmetic:
  rotation   cos and sin in fp32: the angle's last step (2^-24 of at most pi / 4 + 2^-32 turns), the series and its last
             rounding, at most 2^-22.5 in all; two products and a sum in fp32: |error| <= 2^-22 (|a| + |b|) magnitude, and
             half a step of the output's type (bf16: 2^-8 |y|)
  codes      of values: the oracle's, bit for bit.  Of rotated keys: the nearest e4m3 number to a value that is the
             oracle's within the rotation's error
  attention  half a step of bf16 (2^-8 |o|); the two-term weights, 2^-8 sum p |v|, and their floor (half of e4m3's least
             step in units of 1/16, 2^-14, where the largest weight is 2^3 or more), 2^-17 of the largest weight for
             every token; 2^-14 sum p |v| for scores, exponentials and sums in fp32
  lse        2^-16 (1 + |lse|)
"""
import numpy as np
import pytest

from oracle import kv_oracle as K
from paper_2606_26650_gb300 import synthetic as syn
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def device():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def bf16(a, device):
    return U.to_device(syn.round_bf16(np.asarray(a, np.float32)), "bf16", device)


def i32(a, device):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=device)


class Paged:
    """A cache on the host (numpy) and on the GPU with the same content: sequences of `lens` tokens."""

    def __init__(self, r, lens, nkv, page, d, device, max_pages=None, spare=2, kv=None):
        import torch

        from paper_2606_26650_gb300 import catq as C
        need = [-(-n // page) for n in lens]
        width = max_pages or max(max(need), 1)
        self.n_pages, self.page, self.nkv, self.d = sum(need) + spare, page, nkv, d
        order = r.permutation(self.n_pages)
        self.table = np.full((len(lens), width), -7, np.int32)  # what lies behind a sequence's pages is not read
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        # every byte but NaN, in every slot: what lies behind a sequence's last token is finite here
        shape = (self.n_pages, nkv, page, d)
        self.codes = [K.e4m3_encode(np.clip(r.standard_normal(shape) * 100, -448, 448)) for _ in range(2)]
        self.scale = [2.0 ** r.integers(-9, -5, (self.n_pages, nkv)) for _ in range(2)]
        if kv is not None:
            kv(self)
        self.cache = C.KVCache(*(torch.from_numpy(c.copy()).to(device).view(torch.float8_e4m3fn) for c in self.codes),
                               *(torch.tensor(s, dtype=torch.float32, device=device) for s in self.scale),
                               i32(self.table, device))

    def host(self):
        import torch
        c = self.cache
        return ([t.view(torch.uint8).cpu().numpy() for t in (c.k_codes, c.v_codes)],
                [t.cpu().numpy().astype(np.float64) for t in (c.k_scale, c.v_scale)])


def starts(news):
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int32)


def attend(paged, row_start, seq_len, q, nh, device, T=None, with_lse=True, workspace=None, ld_gap=0):
    """catq_kv_attention on bf16-rounded q [T, nh, d]; rows outside every sequence hold 7."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    T = q.shape[0] if T is None else T
    w = nh * paged.d
    Q = torch.full((T, w + ld_gap), 3.0, dtype=torch.bfloat16, device=device)[:, :w]
    Q.copy_(bf16(q.reshape(T, w), device))
    O = torch.full((T, w + ld_gap), 7.0, dtype=torch.bfloat16, device=device)[:, :w]
    lse = torch.full((T, nh), 7.0, dtype=torch.float32, device=device) if with_lse else None
    ws = workspace if workspace is not None else C.kv_attention_workspace(paged.cache, nh)
    C.catq_kv_attention(paged.cache, i32(row_start, device), i32(seq_len, device), Q, O, nh, ws, lse=lse)
    torch.cuda.synchronize()
    assert C.catq_device_status() == 0
    assert not ws[:4096].any()  # the counters are left at zero
    return O.float().cpu().numpy().reshape(T, nh, paged.d).astype(np.float64), lse.cpu().numpy() if with_lse else None


def check_attention(paged, row_start, seq_len, q, nh, got, lse):
    O, want_lse, mag, low = K.attention(*paged.codes, *paged.scale, paged.table, paged.page, row_start, seq_len,
                                        syn.round_bf16(np.asarray(q, np.float32)), q.shape[0], nh)
    outside = np.isnan(want_lse)
    assert (got[outside] == 7).all()
    bound = 2.0 ** -8 * np.abs(O) + (2.0 ** -8 + 2.0 ** -14) * mag + 2.0 ** -17 * low
    off = np.abs(got - O)[~outside] - bound[~outside]
    assert (off <= 0).all(), f"largest excess {off.max():.3g} at bound {bound[~outside].flat[off.argmax()]:.3g}"
    if lse is not None:
        assert (lse[outside] == 7).all()
        a, w = lse[~outside], want_lse[~outside]
        seen = np.isfinite(w)
        assert (a[~seen] == w[~seen]).all()
        assert (np.abs(a[seen] - w[seen]) <= 2.0 ** -16 * (1 + np.abs(w[seen]))).all(), np.abs(a[seen] - w[seen]).max()


@pytest.mark.parametrize("d,nh,nkv,page,lens,news", [
    (128, 8, 8, 64, [1], [1]),                      # one token
    (128, 8, 2, 64, [100], [1]),                    # less than a tile
    (128, 4, 1, 128, [128], [1]),                   # exactly one
    (64, 4, 4, 16, [77], [1]),
    (128, 8, 2, 64, [129, 1, 640, 64], [1, 1, 1, 1]),
    (64, 12, 4, 16, [33, 200, 16, 17, 500], [1, 1, 1, 1, 1]),
    (128, 10, 2, 32, [300, 45], [3, 2]),            # 5 heads a key/value head, drafted tokens: 16 rows a tile
    (128, 32, 8, 16, [260], [4]),                   # 16 rows
    (128, 8, 2, 64, [150, 700], [7, 6]),            # 32 rows
    (64, 6, 2, 32, [190, 400], [9, 8]),
    (128, 8, 2, 64, [300], [300]),                  # a prompt of its own: 64 rows a tile, causal
    (64, 3, 3, 128, [257, 130], [129, 130]),
    (128, 16, 1, 64, [400, 333], [1, 50]),          # 16 heads share one
    (128, 64, 1, 64, [200], [2]),                   # 64 heads share one
    (64, 7, 1, 16, [5, 6, 7, 130], [5, 1, 3, 2]),   # 7 heads share one
    (64, 2, 2, 16, [700, 255, 256, 257], [1, 1, 1, 1]),   # every page size, single tokens and a few
    (64, 2, 2, 32, [700, 255, 256, 257], [1, 1, 1, 1]),
    (64, 2, 1, 64, [700, 31], [1, 1]),
    (64, 2, 1, 128, [129, 600], [1, 1]),
    (128, 2, 2, 16, [500, 127, 128], [1, 1, 1]),
    (128, 2, 1, 32, [500, 33], [1, 1]),
    (128, 2, 2, 128, [500, 1], [1, 1]),
    (64, 4, 1, 32, [300, 77], [4, 3]),
    (64, 4, 1, 128, [300, 77], [3, 4]),
])
def test_attention_matches_oracle(device, d, nh, nkv, page, lens, news):
    r = syn.rng(3, f"kv/{d}/{nh}/{nkv}/{page}/{lens}/{news}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs = starts(news)
    q = r.standard_normal((rs[-1], nh, d)) * 2.0
    got, lse = attend(paged, rs, lens, q, nh, device)
    check_attention(paged, rs, np.array(lens), q, nh, got, lse)


# ------------------------------------------------------------------ rotary positions

def rope_bound(x, freq, interleaved, magnitude):
    """2^-22 (|a| + |b|) magnitude for the elements of a pair, 0 for the others."""
    out = np.zeros(x.shape)
    half = len(freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        out[..., a] = out[..., b] = 2.0 ** -22 * magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,nh,d,rot,interleaved,scaling,gap,far", [
    (1, 1, 128, 128, False, "plain", 0, 1),          # position 0: nothing turns
    (1, 3, 64, 32, True, "plain", 0, 1 << 20),       # far positions
    (67, 5, 128, 128, False, "bands", 64, 131072),   # rows apart
    (33, 9, 128, 64, True, "yarn", 0, 131072),       # part of the head, a magnitude
    (20, 2, 96, 48, False, "linear", 8, 4096),
    (19, 3, 40, 20, False, "plain", 0, 4096),        # sizes off the vector path
    (19, 3, 10, 6, True, "plain", 3, 4096),          # rows of odd alignment
    (300, 32, 64, 64, True, "plain", 0, 2 ** 31 - 1),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope_at_matches_oracle(device, dtype, T, nh, d, rot, interleaved, scaling, gap, far, inverse):
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(4, f"rope/{T}/{nh}/{d}/{rot}")
    kw = dict(factor=8.0, low=1.0, high=32.0 if scaling == "yarn" else 4.0, original=8192.0)
    freq, magnitude = K.frequencies(rot, 500000.0, scaling, **kw)
    rope = C.Rope.create(rot, 500000.0, device, C.ROPE_INTERLEAVED if interleaved else C.ROPE_HALF,
                         ["plain", "linear", "bands", "yarn"].index(scaling), **kw)
    x = r.standard_normal((T, nh, d)).astype(np.float32)
    x = syn.round_bf16(x) if dtype == "bf16" else x
    pos = r.integers(0, far, T)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    whole = torch.full((T, nh * d + gap), 5.0, dtype=dt, device=device)
    X = whole[:, :nh * d]
    X.copy_(U.to_device(x.reshape(T, nh * d), dtype, device))
    Y = torch.empty(T, nh * d, dtype=dt, device=device)
    C.catq_rope_at(X, i32(pos, device), rope, nh, d, Y, inverse=inverse)
    want = K.rope(x, pos, freq, interleaved, magnitude, inverse)
    # positions below 2^31 and turns to 2^-62: the angle is off by 2^-31 turns at most (none of the near ones)
    bound = rope_bound(x, freq, interleaved, magnitude) * (1 + far * 2.0 ** -62 * 2 * np.pi * 2.0 ** 22)
    bound += np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
    got = Y.float().cpu().numpy().reshape(T, nh, d)
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) - bound).max()
    C.catq_rope_at(X, i32(pos, device), rope, nh, d, inverse=inverse)  # in place
    assert torch.equal(X, Y) and (whole[:, nh * d:] == 5).all()
    assert C.catq_device_status() == 0


def test_rope_backward_is_the_gradient(device):
    """<dY, rope(X)> has the gradient rope_at(dY, inverse) in X: against the formula's transpose and central differences
    of the fp64 oracle."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(5, "rope/grad")
    T, nh, d, rot = 7, 2, 32, 16
    freq, magnitude = K.frequencies(rot, 10000.0, "yarn", factor=4.0, low=1.0, high=32.0, original=64.0)
    rope = C.Rope.create(rot, 10000.0, device, C.ROPE_INTERLEAVED, C.ROPE_YARN, factor=4.0, low=1.0, high=32.0,
                         original=64.0)
    x, dy = r.standard_normal((2, T, nh, d))
    dy = dy.astype(np.float32)
    pos = np.arange(T) * 37
    dX = torch.empty(T, nh * d, device=device)
    C.catq_rope_at(U.to_device(dy.reshape(T, -1), "f32", device), i32(pos, device), rope, nh, d, dX, inverse=True)
    got = dX.cpu().numpy().reshape(T, nh, d)
    h = 1e-3
    for at in [(0, 0, 0), (3, 1, 5), (6, 0, 14), (6, 1, 15), (2, 1, 31)]:
        e = np.zeros_like(x)
        e[at] = h
        num = ((K.rope(x + e, pos, freq, True, magnitude) - K.rope(x - e, pos, freq, True, magnitude)) * dy).sum() / (2 * h)
        assert abs(got[at] - num) <= 2.0 ** -21 * magnitude * np.abs(dy[at[:2]]).sum() + 1e-9


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("d,nkv,nh,page,lens,news,rot,interleaved", [
    (128, 2, 4, 64, [1], [1], 128, False),                      # the first token of a sequence
    (128, 2, 2, 64, [64, 65, 130], [1, 1, 1], 128, False),      # the last of a page, the first of one, one inside
    (64, 3, 6, 16, [7, 16, 17, 40, 3], [1, 1, 1, 1, 1], 16, True),
    (128, 1, 5, 128, [200, 128], [150, 128], 128, False),       # whole pages, beginning and ending inside
    (64, 4, 4, 16, [50, 33, 90], [37, 1, 90], 32, True),
    (64, 2, 2, 32, [9, 12], [9, 3], 0, False),                  # no rotation
    (128, 3, 3, 64, [70], [9], 64, True),
    (64, 1, 1, 128, [300, 20], [290, 20], 64, False),
])
@pytest.mark.parametrize("kind", ["normal", "quiet", "growing"])
def test_append_matches_oracle(device, d, nkv, nh, page, lens, news, rot, interleaved, kind):
    """kind: values like the cached ones; far smaller (old scales stay, e4m3's subnormals); far larger (the codes of
    open pages are rounded again)."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(6, f"append/{d}/{nkv}/{page}/{lens}/{news}/{kind}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs, T = starts(news), int(sum(news))
    gain = {"normal": 1.0, "quiet": 2.0 ** -9, "growing": 64.0}[kind]
    k, v = (syn.round_bf16((r.standard_normal((T, nkv, d)) * gain).astype(np.float32)) for _ in range(2))
    v[0, 0] = 0.0  # a row of zeros
    q = syn.round_bf16(r.standard_normal((T, nh, d)).astype(np.float32))
    freq, rope = np.zeros(0), None
    if rot:
        freq, _ = K.frequencies(rot, 10000.0)
        rope = C.Rope.create(rot, 10000.0, device, C.ROPE_INTERLEAVED if interleaved else C.ROPE_HALF)
    fused = torch.empty(T, 2 * nkv * d + 16, dtype=torch.bfloat16, device=device)
    Kt, Vt = fused[:, :nkv * d], fused[:, nkv * d:2 * nkv * d]
    Kt.copy_(bf16(k.reshape(T, -1), device))
    Vt.copy_(bf16(v.reshape(T, -1), device))
    Q = bf16(q.reshape(T, -1), device)
    Qo = torch.empty_like(Q)
    C.catq_kv_append(paged.cache, i32(rs, device), i32(lens, device), Kt, Vt, rope=rope, Q=Q, Q_out=Qo, n_heads=nh)
    torch.cuda.synchronize()
    assert C.catq_device_status() == 0
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, news)])
    codes, scale = paged.host()
    want_q = K.rope(q, pos, freq, interleaved)
    off = np.abs(Qo.float().cpu().numpy().reshape(T, nh, d) - want_q)
    assert (off <= rope_bound(q, freq, interleaved, 1.0) + 2.0 ** -8 * np.abs(want_q)).all()
    K.append(paged.codes[1], paged.scale[1], paged.table, page, rs, lens, v.astype(np.float64))
    assert np.array_equal(scale[1], paged.scale[1])
    assert np.array_equal(K.E4M3[codes[1]], K.E4M3[paged.codes[1]])
    # keys: the nearest code to the rotated value, within the rotation's error; what is not new as the values' codes
    rotated = K.rope(k, pos, freq, interleaved)
    asked = K.append(paged.codes[0], paged.scale[0], paged.table, page, rs, lens, rotated)
    assert np.array_equal(scale[0], paged.scale[0])
    new = ~np.isnan(asked)
    assert np.array_equal(K.E4M3[codes[0]][~new], K.E4M3[paged.codes[0]][~new])
    slack = np.full(codes[0].shape, np.nan)
    err, r0 = rope_bound(k, freq, interleaved, 1.0), 0
    for b, (n, m) in enumerate(zip(lens, news)):
        for i in range(m):
            p, at = paged.table[b][(n - m + i) // page], (n - m + i) % page
            slack[p, :, at] = err[r0 + i] / np.maximum(scale[0][p], 1e-300)[:, None]
        r0 += m
    got = K.E4M3[codes[0]][new]
    assert (np.abs(got - asked[new]) <= K.half_step(asked[new]) * (1 + 2.0 ** -20) + slack[new]).all()


@pytest.mark.parametrize("d,nkv,nh,page,lens,news", [
    # single tokens, idle slots and a long prompt among them; more sequences than a CTA has threads
    (128, 2, 4, 64, [90, 0, 17] * 100 + [700] + [64, 129], [1, 0, 1] * 100 + [650] + [1, 1]),
    (64, 1, 2, 16, [3, 30, 64, 7] * 150, [0, 1, 2, 3] * 150),
    # more pages than CTAs: a CTA's run of them begins and ends inside a page's heads
    (128, 3, 3, 32, [2500, 1700, 40], [2480, 1700, 17]),
    (128, 4, 1, 128, [5000, 3], [4980, 3]),
    (64, 5, 5, 64, [3333, 2000], [3333, 1993]),
    (128, 5, 5, 16, [1234, 900], [1230, 900]),
])
@pytest.mark.parametrize("kind", ["normal", "growing"])
def test_append_of_mixed_batches(device, d, nkv, nh, page, lens, news, kind):
    test_append_matches_oracle(device, d, nkv, nh, page, lens, news, d // 2, False, kind)


def test_append_then_attention_then_packed_linear(device):
    """Decoding as it is used: a prompt of unequal lengths is appended, then tokens one by one, each with attention over
    the cache and the packed output projection; the oracle walks its own cache beside it."""
    import torch

    from oracle import catq_oracle as O
    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(7, "kv/loop")
    nh, nkv, d, page, B, H, g = 8, 2, 64, 16, 3, 192, 128
    N, Kdim = H, nh * d
    W = syn.round_bf16(r.standard_normal((N, Kdim)).astype(np.float32) * 0.02)
    layer = C.Layer.create(U.to_device(W, "bf16", device), g)
    C.catq_group_stats(layer)
    codes = torch.empty(N * Kdim // 4, dtype=torch.uint8, device=device)
    alpha = torch.empty(N * Kdim // g, dtype=torch.float32, device=device)
    C.catq_hard_ternarize_pack(layer, codes, alpha)
    freq, _ = K.frequencies(d, 10000.0)
    rope = C.Rope.create(d, 10000.0, device)
    prompt = np.array([21, 5, 40])
    steps = 4
    paged = Paged(r, prompt + steps, nkv, page, d, device)
    lens = i32(prompt, device)
    ws = C.kv_attention_workspace(paged.cache, nh)
    for step in range(steps + 1):
        news = prompt if step == 0 else np.ones(3, np.int64)
        now = prompt + step
        rs, T = starts(news), int(news.sum())
        q, k, v = (syn.round_bf16(r.standard_normal((T, h, d)).astype(np.float32)) for h in (nh, nkv, nkv))
        Q = bf16(q.reshape(T, -1), device)
        Kt, Vt = bf16(k.reshape(T, -1), device), bf16(v.reshape(T, -1), device)
        if step:
            lens += 1
        row_start = i32(rs, device)
        C.catq_kv_append(paged.cache, row_start, lens, Kt, Vt, rope=rope, Q=Q, n_heads=nh)
        A = torch.empty(T, nh * d, dtype=torch.bfloat16, device=device)
        C.catq_kv_attention(paged.cache, row_start, lens, Q, A, nh, ws)
        last = A[[int(e) - 1 for e in rs[1:]]].contiguous()
        Y = torch.empty(B, N, dtype=torch.bfloat16, device=device)
        C.catq_ternary_infer(codes, alpha, N, Kdim, g, last, Y)
        torch.cuda.synchronize()
        assert C.catq_device_status() == 0
        pos = np.concatenate([np.arange(n - m, n) for n, m in zip(now, news)])
        K.append(paged.codes[0], paged.scale[0], paged.table, page, rs, now, K.rope(k, pos, freq, False))
        K.append(paged.codes[1], paged.scale[1], paged.table, page, rs, now, v.astype(np.float64))
        assert np.array_equal(K.E4M3[paged.host()[0][1]], K.E4M3[paged.codes[1]])
        paged.codes[0], paged.scale[0] = paged.host()[0][0], paged.host()[1][0]  # a key on a border may differ
        want, _, _, _ = K.attention(*paged.codes, *paged.scale, paged.table, page, rs, now,
                                    Q.float().cpu().numpy().reshape(T, nh, d), T, nh)
        assert U.fro_rel(A.float().cpu().numpy(), want.reshape(T, -1)) <= 2.0 ** -7
        want_y = O.ternary_infer(U.to_host(codes), U.to_host(alpha), N, Kdim, g, U.to_host(last))
        assert U.fro_rel(U.to_host(Y), want_y) <= U.TOL_BF16


# ------------------------------------------------------------------ what the calls allow and ordinary cases do not show

@pytest.mark.parametrize("d,nh,nkv,page,lens,news", [
    (128, 4, 1, 64, [5000], [1]),                   # one sequence over many runs, whose parts are joined
    (64, 2, 1, 32, [9000, 20], [1, 1]),
    (128, 8, 2, 32, [1500, 900], [700, 3]),         # many rows a key/value head
    (128, 5, 1, 16, [2100], [130]),
    (64, 4, 2, 64, [1100], [200]),
    (128, 24, 1, 128, [3000], [1]),                 # 24 heads share one, split
])
def test_long_attention_matches_oracle(device, d, nh, nkv, page, lens, news):
    r = syn.rng(8, f"kvlong/{d}/{nh}/{nkv}/{lens}/{news}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs = starts(news)
    q = r.standard_normal((rs[-1], nh, d)) * 2.0
    got, lse = attend(paged, rs, lens, q, nh, device)
    check_attention(paged, rs, np.array(lens), q, nh, got, lse)
    again, _ = attend(paged, rs, lens, q, nh, device, with_lse=False)
    assert np.array_equal(got, again)  # the same bits


@pytest.mark.parametrize("d,news", [(128, [1, 0, 1, 2, 1]), (64, [1, 0, 1, 2, 1]), (128, [1, 0, 1, 90, 1])])
def test_idle_slots_and_rows_outside(device, d, news):
    """A sequence without rows, one whose row sees nothing (length 0), one shorter than its rows, rows behind the last."""
    r = syn.rng(9, f"idle/{d}")
    lens = [40, 33, 0, 1 if news[3] == 2 else 50, 70]
    paged = Paged(r, lens, 2, 32, d, device, max_pages=4)
    rs = starts(news)
    T = int(rs[-1]) + 3
    q = r.standard_normal((T, 4, d))
    got, lse = attend(paged, rs, lens, q, 4, device, ld_gap=16)
    check_attention(paged, rs, np.array(lens), q, 4, got, lse)


@pytest.mark.parametrize("d,new", [(128, 1), (64, 1), (128, 3), (64, 20), (128, 60)])
def test_bytes_behind_the_last_token_do_not_count(device, d, new):
    """Every byte of the pages behind the last token, NaN codes among them."""
    import torch
    r = syn.rng(10, f"behind/{d}/{new}")
    lens = [new + 70, new + 129]
    paged = Paged(r, lens, 2, 64, d, device)
    for c in (paged.cache.k_codes, paged.cache.v_codes):
        raw = c.view(torch.uint8)
        for b, n in enumerate(lens):
            raw[int(paged.table[b][n // 64]), :, n % 64:] = 0x7F
    rs = starts([new, new])
    q = r.standard_normal((rs[-1], 4, d))
    got, lse = attend(paged, rs, lens, q, 4, device)
    check_attention(paged, rs, np.array(lens), q, 4, got, lse)


@pytest.mark.parametrize("d,new", [(128, 4), (64, 4), (128, 80), (64, 40)])
def test_values_that_are_not_finite(device, d, new):
    """An infinite key and a NaN value: the pages' scales are NaN, the rows that see them NaN and no other; a row whose
    query is not finite is NaN by itself."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(11, f"nonfinite/{d}/{new}")
    page, nkv, nh, n = 16, 2, 4, 90
    paged = Paged(r, [n, n, n], nkv, page, d, device)
    rs = starts([new] * 3)
    T = 3 * new
    k, v = (syn.round_bf16(r.standard_normal((T, nkv, d)).astype(np.float32)) for _ in range(2))
    bad = n - new + new // 2  # the position in sequences 0 (key of head 1) and 1 (value of head 0)
    k[new // 2, 1, 3] = np.inf
    v[new + new // 2, 0, 5] = np.nan
    q = syn.round_bf16(r.standard_normal((T, nh, d)).astype(np.float32))
    q[2 * new + 1, 2, 0] = np.nan
    Q = bf16(q.reshape(T, -1), device)
    rope = None
    C.catq_kv_append(paged.cache, i32(rs, device), i32([n] * 3, device), bf16(k.reshape(T, -1), device),
                     bf16(v.reshape(T, -1), device), rope=rope)
    O = torch.empty_like(Q)
    C.catq_kv_attention(paged.cache, i32(rs, device), i32([n] * 3, device), Q, O, nh,
                        C.kv_attention_workspace(paged.cache, nh))
    torch.cuda.synchronize()
    assert C.catq_device_status() == 0
    codes, scale = paged.host()
    K.append(paged.codes[0], paged.scale[0], paged.table, page, rs, [n] * 3, k.astype(np.float64))
    K.append(paged.codes[1], paged.scale[1], paged.table, page, rs, [n] * 3, v.astype(np.float64))
    for got, want in zip(scale, paged.scale):
        assert np.array_equal(got, want, equal_nan=True)
    assert np.isnan(scale[0]).sum() == 1 and np.isnan(scale[1]).sum() == 1
    got = O.float().cpu().numpy().reshape(3, new, nh, d)
    sees = (n - new + np.arange(new)) >= bad // page * page
    want_nan = np.zeros((3, new, nh), bool)
    want_nan[0, sees, 2:] = True
    want_nan[1, sees, :2] = True
    want_nan[2, 1, 2] = True
    assert np.array_equal(np.isnan(got).all(-1), want_nan) and np.array_equal(np.isnan(got).any(-1), want_nan)


def test_a_recycled_page_forgets_its_scale(device):
    """A NaN or huge scale of a page's last use does not outlive its first token's append."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(12, "recycled")
    paged = Paged(r, [17], 1, 16, 64, device)
    paged.cache.k_scale[int(paged.table[0][1])] = float("nan")
    paged.cache.v_scale[int(paged.table[0][1])] = 1e20
    k = bf16(r.standard_normal((1, 64)), device)
    C.catq_kv_append(paged.cache, i32([0, 1], device), i32([17], device), k, k)
    torch.cuda.synchronize()
    want = K.scale_of(float(k.float().abs().max()))
    assert paged.cache.k_scale[int(paged.table[0][1])].item() == want
    assert paged.cache.v_scale[int(paged.table[0][1])].item() == want


@pytest.mark.parametrize("d,new", [(128, 1), (64, 1), (128, 6), (128, 70), (64, 30)])
@pytest.mark.parametrize("gain", [3e4, 1e30])
def test_large_scores_pick_one_token(device, d, new, gain):
    """Scores far apart (2^24 and more): the weight of the largest is 1, whatever the others'."""
    r = syn.rng(13, f"large/{d}/{new}")
    lens = [new + 300]
    paged = Paged(r, lens, 1, 64, d, device)
    q = r.standard_normal((new, 2, d)) * gain
    got, _ = attend(paged, starts([new]), lens, q, 2, device)
    qr = syn.round_bf16(np.asarray(q, np.float32)).astype(np.float64)
    for i in range(new):
        n = lens[0] - new + i + 1
        pages = [paged.table[0][j] for j in range(-(-n // 64))]
        kc, vc = (np.concatenate([K.E4M3[c[p, 0]] * s[p, 0] for p in pages])[:n] for c, s in
                  ((paged.codes[0], paged.scale[0]), (paged.codes[1], paged.scale[1])))
        for h in range(2):
            score = kc @ qr[i, h]
            best = np.argsort(score)[-2:]
            if score[best[1]] - score[best[0]] > 1e-4 * np.abs(score).max():  # (fp32 tells them apart)
                assert np.allclose(got[i, h], vc[best[1]], rtol=2.0 ** -7, atol=0)


def test_output_over_the_queries_and_strided_rows(device):
    import torch

    from paper_2606_26650_gb300 import catq as C
    for d, new in ((128, 2), (64, 2), (128, 50)):
        r = syn.rng(14, f"inplace/{d}/{new}")
        lens = [new + 200, new + 3]
        paged = Paged(r, lens, 2, 32, d, device)
        rs = starts([new, new])
        q = r.standard_normal((2 * new, 4, d))
        want, _ = attend(paged, rs, lens, q, 4, device)
        whole = torch.full((2 * new, 4 * d + 32), 9.0, dtype=torch.bfloat16, device=device)
        Q = whole[:, 16:16 + 4 * d]
        Q.copy_(bf16(q.reshape(2 * new, -1), device))
        C.catq_kv_attention(paged.cache, i32(rs, device), i32(lens, device), Q, Q, 4,
                            C.kv_attention_workspace(paged.cache, 4))
        torch.cuda.synchronize()
        assert np.array_equal(Q.float().cpu().numpy().reshape(want.shape), want)
        assert (whole[:, :16] == 9).all() and (whole[:, 16 + 4 * d:] == 9).all()


def test_bad_pages_offsets_and_lengths_are_latched(device):
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(15, "bad")
    for d, new in ((128, 1), (64, 1), (128, 40)):
        lens = np.array([new + 60, new + 60, new + 60, new + 60])
        paged = Paged(r, lens, 2, 32, d, device, max_pages=4)
        rs = starts([new] * 4)
        T = int(rs[-1])
        q = r.standard_normal((T, 4, d))
        want, _ = attend(paged, rs, lens, q, 4, device)
        ws = C.kv_attention_workspace(paged.cache, 4)
        Q = bf16(q.reshape(T, -1), device)

        def call(row_start, seq_len):
            O = torch.full_like(Q, 7.0)
            C.catq_kv_attention(paged.cache, i32(row_start, device), i32(seq_len, device), Q, O, 4, ws)
            status = C.catq_device_status()
            assert C.catq_device_status() == 0 and not ws[:4096].any()
            return status, O.float().cpu().numpy().reshape(T, 4, d)

        # pages that do not exist count as zeros: keys and values of that page 0
        table = paged.cache.table.clone()
        for sick in (-1, paged.n_pages, 2 ** 31 - 1, -2 ** 31):
            paged.cache.table[1, 1] = sick
            status, got = call(rs, lens)
            assert C.STATUS[status] == "CATQ_ERR_INDEX"
            keep = [i for i in range(T) if not new <= i < 2 * new]
            assert np.array_equal(got[keep], want[keep])
            zero = Paged.__new__(Paged)
            zero.__dict__.update(paged.__dict__)
            zero.codes, zero.scale = [c.copy() for c in paged.codes], [s.copy() for s in paged.scale]
            p = paged.table[1][1]
            for c in zero.codes:
                c[p] = 0
            one = slice(new, 2 * new)
            ref, _, mag, low = K.attention(*zero.codes, *zero.scale, [paged.table[1]], 32, [0, new], lens[1:2],
                                           syn.round_bf16(np.asarray(q[one], np.float32)), new, 4)
            assert (np.abs(got[one] - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -14) * mag
                    + 2.0 ** -17 * low).all()
            if new == 1:  # and nothing is appended to them (position 33 of sequence 1 is the only one)
                before = paged.host()
                kv = bf16(r.standard_normal((T, 2 * d)), device)
                C.catq_kv_append(paged.cache, i32(rs, device), i32(np.array([0, 34, 0, 0]), device), kv, kv)
                assert C.STATUS[C.catq_device_status()] == "CATQ_ERR_INDEX"
                after = paged.host()
                assert all(np.array_equal(x, y) for x, y in zip(before[0] + before[1], after[0] + after[1]))
            paged.cache.table.copy_(table)
        # offsets that fall, reach past the rows or begin before them; lengths that do not fit the table
        for row_start, seq_len, lost in [
                (np.array([0, new, new - 1, 3 * new, 4 * new]), lens, [1, 2]),
                (np.array([0, new, 2 * new, 3 * new, 4 * new + 1]), lens, [3]),
                (np.array([-1, new, 2 * new, 3 * new, 4 * new]), lens, [0]),
                (rs, np.array([lens[0], -1, lens[2], lens[3]]), [1]),
                (rs, np.array([lens[0], lens[1], 129, lens[3]]), [2])]:
            status, got = call(row_start, seq_len)
            assert C.STATUS[status] == "CATQ_ERR_INDEX"
            for b in range(4):
                # (offsets 0, new, new - 1, 3 new: sequence 2 by itself is in order and has row new - 1 too, the last of
                # sequence 0, so nothing is said about that one)
                rows = slice(b * new, (b + 1) * new - (b == 0 and lost == [1, 2]))
                if b not in lost:
                    assert np.array_equal(got[rows], want[rows])
                elif lost != [1, 2]:  # (sequence 2's rows there: new - 1 .. 3 new - 1, all of sequence 1's among them)
                    assert (got[rows] == 7).all()


@pytest.mark.parametrize("d", [128, 64])
def test_a_batch_in_two_calls(device, d):
    """Single tokens and prompts of one batch by a call each, on slices of the offsets, lengths and table."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(14, f"attn/two/{d}")
    lens, news = [40, 300, 1, 120, 270], [1, 1, 1, 77, 33]
    paged = Paged(r, lens, 2, 16, d, device)
    rs, nh, T = starts(news), 8, sum(news)
    q = syn.round_bf16(r.standard_normal((T, nh, d)).astype(np.float32))
    Q, offsets, lengths = bf16(q.reshape(T, -1), device), i32(rs, device), i32(lens, device)
    O = torch.full((T, nh * d), 7.0, dtype=torch.bfloat16, device=device)
    lse = torch.full((T, nh), 7.0, device=device)
    c = paged.cache
    ws = C.kv_attention_workspace(c, nh)
    for b0, b1 in ((0, 3), (3, 5)):
        part, end = C.KVCache(c.k_codes, c.v_codes, c.k_scale, c.v_scale, c.table[b0:b1]), int(rs[b1])
        C.catq_kv_attention(part, offsets[b0:b1 + 1], lengths[b0:b1], Q[:end], O[:end], nh, ws, lse[:end])
        if b0 == 0:
            assert (O[3:] == 7).all() and (lse[3:] == 7).all()
    assert C.catq_device_status() == 0
    check_attention(paged, rs, lens, q, nh, O.float().cpu().numpy().reshape(T, nh, d), lse.cpu().numpy())


def test_many_sequences(device):
    """More sequences than the kernels have threads, many of them empty."""
    r = syn.rng(16, "many")
    B = 1500
    lens = r.integers(0, 40, B)
    news = np.minimum(r.integers(0, 2, B), lens)
    for d in (128, 64):
        paged = Paged(r, list(lens), 1, 16, d, device)
        rs = starts(news)
        q = r.standard_normal((rs[-1], 2, d))
        got, lse = attend(paged, rs, lens, q, 2, device)
        check_attention(paged, rs, lens, q, 2, got, lse)


def test_offsets_past_32_bits(device):
    """Caches of more than 2^32 bytes, the sequence's pages at their end."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(17, "far")
    for d, new in ((128, 1), (64, 2), (128, 40)):
        n_pages, page, n = 5 * 2 ** 30 // (64 * d), 64, 200
        table = np.array([[n_pages - 1 - 7 * i for i in range(4)]], np.int32)
        kc, vc = (torch.empty(n_pages, 1, page, d, dtype=torch.uint8, device=device) for _ in range(2))
        ks, vs = (torch.ones(n_pages, 1, device=device) for _ in range(2))
        cache = C.KVCache(kc.view(torch.float8_e4m3fn), vc.view(torch.float8_e4m3fn), ks, vs, i32(table, device))
        k, v = (syn.round_bf16(r.standard_normal((n, 1, d)).astype(np.float32)) for _ in range(2))
        C.catq_kv_append(cache, i32([0, n], device), i32([n], device), bf16(k.reshape(n, d), device),
                         bf16(v.reshape(n, d), device))
        q = r.standard_normal((new, 2, d))
        Q = bf16(q.reshape(new, -1), device)
        O = torch.empty_like(Q)
        C.catq_kv_attention(cache, i32([0, new], device), i32([n], device), Q, O, 2, C.kv_attention_workspace(cache, 2))
        torch.cuda.synchronize()
        assert C.catq_device_status() == 0
        small = [np.zeros((4, 1, page, d), np.uint8) for _ in range(2)]
        scale = [np.zeros((4, 1)) for _ in range(2)]
        for c, s, x in zip(small, scale, (k, v)):
            K.append(c, s, [[0, 1, 2, 3]], page, [0, n], [n], x.astype(np.float64))
        for c, t in zip(small, (kc, vc)):
            got = t[torch.tensor(table[0], device=device).long()].cpu().numpy()
            assert np.array_equal(K.E4M3[got].reshape(-1, d)[:n], K.E4M3[c].reshape(-1, d)[:n])
        ref, _, mag, low = K.attention(*small, *scale, [[0, 1, 2, 3]], page, [0, new], [n],
                                       syn.round_bf16(np.asarray(q, np.float32)), new, 2)
        got = O.float().cpu().numpy().reshape(new, 2, d)
        assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -14) * mag + 2.0 ** -17 * low).all()
        del kc, vc, ks, vs, cache
        torch.cuda.empty_cache()


def test_a_captured_step_follows_the_lengths(device):
    """Append and attention captured once, replayed as the sequences grow: lengths and rows are read on the device."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    for d in (128, 64):
        r = syn.rng(18, f"graph/{d}")
        B, nh, nkv, page, steps = 3, 4, 2, 16, 40
        paged, eager = (Paged(syn.rng(18, f"graph/cache/{d}"), [5 + steps, 14 + steps, 31 + steps], nkv, page, d, device)
                        for _ in range(2))
        rope = C.Rope.create(d, 10000.0, device)
        lens = i32([5, 14, 31], device)
        rs = i32([0, 1, 2, 3], device)
        K_, V, Q, O = (torch.zeros(B, h * d, dtype=torch.bfloat16, device=device) for h in (nkv, nkv, nh, nh))
        ws = C.kv_attention_workspace(paged.cache, nh)

        def step(cache, ws):
            C.catq_kv_append(cache, rs, lens, K_, V, rope=rope, Q=Q, n_heads=nh)
            C.catq_kv_attention(cache, rs, lens, Q, O, nh, ws)

        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        start_lens = lens.clone()
        with torch.cuda.stream(side):
            step(paged.cache, ws)
            side.synchronize()
            with torch.cuda.graph(graph, stream=side):
                step(paged.cache, ws)
        torch.cuda.synchronize()
        # the warm-up appended zeros at the first position: begin again from the same caches
        for t in ("k_codes", "v_codes", "k_scale", "v_scale"):
            getattr(paged.cache, t).view(torch.uint8 if "codes" in t else torch.float32).copy_(
                getattr(eager.cache, t).view(torch.uint8 if "codes" in t else torch.float32))
        lens.copy_(start_lens)
        ws2 = C.kv_attention_workspace(eager.cache, nh)
        for i in range(steps):
            k, v, q = (bf16(r.standard_normal((B, h * d)), device) for h in (nkv, nkv, nh))
            outs = []
            for run in (lambda: graph.replay(), lambda: step(eager.cache, ws2)):
                K_.copy_(k), V.copy_(v), Q.copy_(q)
                run()
                outs.append(O.clone())
            lens += 1
            assert torch.equal(outs[0], outs[1]), i
        torch.cuda.synchronize()
        assert C.catq_device_status() == 0


def test_two_streams_with_workspaces_of_their_own(device):
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(19, "streams")
    jobs = []
    for d, nh, nkv, lens, news in ((128, 8, 2, [3000, 700], [1, 1]), (64, 4, 4, [900, 50], [2, 1]),
                                   (128, 4, 1, [1200], [100])):
        paged = Paged(r, lens, nkv, 32, d, device)
        rs = starts(news)
        Q = bf16(r.standard_normal((rs[-1], nh * d)), device)
        jobs.append((paged, i32(rs, device), i32(lens, device), Q, torch.empty_like(Q), nh,
                     C.kv_attention_workspace(paged.cache, nh), torch.cuda.Stream()))
    want = []
    for p, rs, sl, Q, O, nh, ws, _ in jobs:
        C.catq_kv_attention(p.cache, rs, sl, Q, O, nh, ws)
        want.append(O.clone())
    torch.cuda.synchronize()
    for _ in range(20):
        for p, rs, sl, Q, O, nh, ws, st in jobs:
            O.zero_()
        torch.cuda.synchronize()
        for p, rs, sl, Q, O, nh, ws, st in jobs:
            C.catq_kv_attention(p.cache, rs, sl, Q, O, nh, ws, stream=st)
        torch.cuda.synchronize()
        for (_, _, _, _, O, _, _, _), w in zip(jobs, want):
            assert torch.equal(O, w)
    assert C.catq_device_status() == 0
