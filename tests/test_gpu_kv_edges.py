"""GPU tests of the decoding calls at the ends of their ranges, against the fp64 oracle: rows of more than 2^31 elements, launches
that overlap, sines and cosines by themselves, weights far below a row's largest, tiny queries,
pages of zeros, rows before a sequence's first position.

Tolerances, from the arithmetic: a rotation is off by 2^-22 (|a| + |b|) (sine and cosine within 2^-22.5, two products and a
sum in fp32) and half a step of the output's type."""
import numpy as np
import pytest

from oracle import kv_oracle as K
from paper_2606_26650_gb300 import synthetic as syn
from tests.test_gpu_kv import Paged, attend, bf16, check_attention, device, i32, rope_bound, starts  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_of_rows_past_32_bits(device, dtype):  # noqa: F811
    """One row of 40000 heads of 65536: a head's offset passes 2^31 elements from head 32768 on."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    nh, d, rot, pos = 40000, 65536, 64, 12345
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device=device).manual_seed(5)
    X = torch.empty(1, nh * d, dtype=dt, device=device).normal_(generator=gen)
    rope = C.Rope.create(rot, 10000.0, device)
    Y = torch.zeros_like(X)
    C.catq_rope_at(X, i32([pos], device), rope, nh, d, Y)
    x, y = X.view(nh, d), Y.view(nh, d)
    assert torch.equal(x[:, rot:], y[:, rot:])  # what is not rotated passes unchanged
    freq, _ = K.frequencies(rot, 10000.0)
    host = x[:, :rot].float().cpu().numpy()[None].astype(np.float64)
    want = K.rope(host, np.array([pos]), freq, False)
    bound = rope_bound(host, freq, False, 1.0) + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
    got = y[:, :rot].float().cpu().numpy()[None]
    assert (np.abs(got - want) <= bound).all()
    C.catq_rope_at(X, i32([pos], device), rope, nh, d)  # in place
    assert torch.equal(X, Y)
    assert C.catq_device_status() == 0
    del X, Y, x, y
    torch.cuda.empty_cache()


@pytest.mark.parametrize("shift", [0, 8])
def test_a_decode_step_sees_what_the_launch_ahead_wrote(device, shift):  # noqa: F811
    """Append, attention over its own queries and the packed output projection, back to back, every launch resident while the one
    ahead runs: the same bits as with a wait between them.  shift: rows of 32-byte and of 16-byte alignment."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    nh, nkv, d, page, B, g, steps = 16, 4, 64, 16, 5, 128, 24
    N, kdim = 512, nh * d
    gen = torch.Generator(device=device).manual_seed(11)

    def normal(*shape):
        return torch.empty(*shape, dtype=torch.bfloat16, device=device).normal_(generator=gen)

    codes = torch.randint(0, 255, (N * kdim // 4,), dtype=torch.uint8, device=device, generator=gen) & 0b01010101
    alpha = torch.rand(N * kdim // g, device=device, generator=gen)
    rope = C.Rope.create(d, 10000.0, device)
    tokens = [(normal(B, nh * d), normal(B, nkv * d), normal(B, nkv * d)) for _ in range(steps)]
    results = []
    for wait in (True, False):
        table = torch.arange(B * 4, dtype=torch.int32, device=device).view(B, 4)
        cache = C.KVCache.create(B * 4, nkv, page, d, table)
        ws = C.kv_attention_workspace(cache, nh)
        rows = i32(np.arange(B + 1), device)
        lens = [i32(np.arange(B) * 7 + i + 1, device) for i in range(steps)]
        flat = torch.zeros(B * nh * d + 16, dtype=torch.bfloat16, device=device)
        Q = flat[shift:shift + B * nh * d].view(B, nh * d)
        out = [torch.empty(B, N, dtype=torch.bfloat16, device=device) for _ in range(steps)]
        torch.cuda.synchronize()
        for i, (q, k, v) in enumerate(tokens):
            Q.copy_(q)
            for call in (lambda: C.catq_kv_append(cache, rows, lens[i], k, v, rope=rope, Q=Q, n_heads=nh),
                         lambda: C.catq_kv_attention(cache, rows, lens[i], Q, Q, nh, ws),
                         lambda: C.catq_ternary_infer(codes, alpha, N, kdim, g, Q, out[i])):
                call()
                if wait:
                    torch.cuda.synchronize()
        torch.cuda.synchronize()
        assert C.catq_device_status() == 0
        results.append(torch.stack(out))
    assert torch.isfinite(results[0].float()).all()
    assert torch.equal(results[0], results[1])


@pytest.mark.parametrize("pos", [1, -1, 2 ** 31 - 1])
def test_sine_and_cosine_by_themselves(device, pos):  # noqa: F811
    """(1, 0) rotated by a million angles from all around the circle, those at the quarter turns more densely: cosine and sine to
    2^-22.5.  (The angle's last step, 2^-32 of a turn, is 2^-29.3.)"""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = np.random.default_rng(22)
    half, nh = 32768, 1
    X = torch.zeros(1, 2 * half, device=device)
    X[:, :half] = 1.0
    for i in range(32):
        turns = r.integers(0, 2 ** 64, half, dtype=np.uint64)
        if i % 2:  # within 2^-4 of a quarter turn
            turns = (turns >> np.uint64(4)) + (turns & np.uint64(3)) * np.uint64(2 ** 62) - np.uint64(2 ** 59)
        rope = C.Rope(torch.from_numpy(turns.view(np.int64).copy()).to(device), 2 * half)
        Y = torch.empty_like(X)
        C.catq_rope_at(X, i32([pos], device), rope, nh, 2 * half, Y)
        got = Y.cpu().numpy().reshape(2, half).astype(np.float64)
        with np.errstate(over="ignore"):
            part = turns * np.uint64(pos % 2 ** 64)  # modulo one turn
        angle = part.astype(np.longdouble) * (2 * np.pi / np.longdouble(2) ** 64)
        assert np.abs(got[0] - np.cos(angle)).max() <= 2.0 ** -22.5
        assert np.abs(got[1] - np.sin(angle)).max() <= 2.0 ** -22.5
    assert C.catq_device_status() == 0


class LoudAndTail:
    """A token (at position `loud`) far above n - 1 others, whose scores spread by 0.3 nats; every key/value head holds the
    same, every query head of a group has its own others.  Values: one constant an element, or (silent) a spread around it and nothing
    for the loud token.  The loud token's key has only the first element, the others' keys all but that, so that a query's
    first element alone says how far it is above them."""
    page = 128

    def __init__(self, r, d, n, new, group, nkv, loud, device):
        import torch
        self.n, self.d, self.new, self.group, self.loud, self.device = n, d, new, group, loud, device
        n_pages = -(-n // self.page)
        k = r.standard_normal((n_pages * self.page, d))
        k[:, 0] = 0.0
        k[loud] = 0.0
        k[loud, 0] = 16.0
        v = np.tile(np.linspace(1.0, 1.75, d), (n_pages * self.page, 1))
        w = v * (1 + 0.25 * r.standard_normal(v.shape).clip(-3, 3))
        w[loud] = 0.0
        kc, *vc = (K.e4m3_encode(x) for x in (k, v, w))

        def pages(c):
            c = torch.from_numpy(c.reshape(n_pages, 1, self.page, d)).to(device)
            return c.expand(-1, nkv, -1, -1).contiguous().view(torch.float8_e4m3fn)

        self.keys, self.values = pages(kc), [pages(c) for c in vc]
        self.ones = torch.ones(n_pages, nkv, device=device)
        self.q = syn.round_bf16((0.3 * r.standard_normal((new, group, d))).astype(np.float32)).astype(np.float64)
        rows = new * group
        last = n - new + np.arange(new).repeat(group)
        x = self.q.reshape(rows, d) @ K.E4M3[kc[:n]].T / np.sqrt(d)
        x[np.arange(n)[None] > last[:, None]] = -np.inf
        x[:, loud] = -np.inf
        e = np.exp(x)
        self.others = e.sum(axis=1).reshape(new, group)
        self.sums = [(e @ K.E4M3[c[:n]]).reshape(new, group, d) for c in vc]
        self.loud_value = [K.E4M3[c[loud]] for c in vc]

    def case(self, gap, silent):
        """Queries whose loud token weighs about 2^gap of another; output and log-sum-exp in fp64."""
        q0 = syn.round_bf16(np.float32([gap * np.log(2) * np.sqrt(self.d) / 16.0]))[0]
        q = self.q.copy()
        q[..., 0] = q0
        top = np.exp(float(q0) * 16.0 / np.sqrt(self.d))
        total = self.others + top
        return q, (self.sums[silent] + top * self.loud_value[silent]) / total[..., None], np.log(total)

    def cache(self, B, silent):
        from paper_2606_26650_gb300 import catq as C
        table = np.tile(np.arange(self.keys.shape[0], dtype=np.int32), (B, 1))
        return C.KVCache(self.keys, self.values[silent], self.ones, self.ones, i32(table, self.device))


@pytest.mark.parametrize("d,new,group", [
    (128, 1, 1), (128, 2, 4), (128, 4, 4), (128, 7, 4), (128, 16, 4), (128, 32, 4), (128, 40, 5),
    (64, 1, 1), (64, 4, 4), (64, 8, 4), (64, 33, 4)])
@pytest.mark.parametrize("n,B,nkv,loud", [(8192, 40, 8, 3), (131072, 40, 8, 3), (8192, 2, 2, 5000)])
def test_the_tail_below_a_loud_token_counts(device, d, new, group, n, B, nkv, loud):  # noqa: F811
    """One token far above thousands of others, whose weights count by their sum: the output is the constant that all values are, or,
    where the loud token's value is nothing, what the others give.  A bound that does not grow with the number of tokens: half a
    step of bf16 (2^-8); the loud weight is a power of two and exact, the others' errors, 2^-9 at most and of either sign, come to
    less than 2^-11 over thousands; what is below their range is 2^-31 of the largest (2^-11 of a weight of 2^-20; of a constant's
    131,072 terms 2^-14); scores, exponentials and sums 2^-12: 2^-8 + 2^-9 of the output, all of whose terms have one sign.
    With 40 sequences on the same pages whole rows fall to one CTA; few sequences are cut, long ones in pieces."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    t = LoudAndTail(syn.rng(23, f"tail/{d}/{new}/{group}/{n}"), d, n, new, group, nkv, loud, device)
    row_start, seq_len = i32(np.arange(B + 1) * new, device), i32([n] * B, device)
    for silent, gaps in ((0, (14, 16.4, 17.3, 18, 20, 22, 24)), (1, (12, 16, 18, 20))):
        cache = t.cache(B, silent)
        ws = C.kv_attention_workspace(cache, nkv * group)
        for gap in gaps:
            q, want, want_lse = t.case(gap, silent)
            Q = bf16(np.tile(q[:, None], (B, nkv, 1, 1)).reshape(B * new, nkv * group * d), device)
            O = torch.empty_like(Q)
            lse = torch.empty(B * new, nkv * group, device=device)
            C.catq_kv_attention(cache, row_start, seq_len, Q, O, nkv * group, ws, lse)
            got = O.float().cpu().numpy().reshape(B, new, nkv, group, d)
            off = np.abs(got / want[None, :, None] - 1).max()
            assert off <= 2.0 ** -8 + 2.0 ** -9, (gap, silent, f"2^{np.log2(off):.2f}")
            off = np.abs(lse.cpu().numpy().reshape(B, new, nkv, group) - want_lse[None, :, None]).max()
            assert off <= 2.0 ** -16 * (1 + want_lse.max())
    assert C.catq_device_status() == 0


@pytest.mark.parametrize("d,new", [(128, 1), (64, 1), (128, 6), (64, 20), (128, 60)])
def test_tiny_queries_against_huge_keys(device, d, new):  # noqa: F811
    """Queries of 2^-117 and keys of 2^118: the scores are ordinary ones."""
    r = syn.rng(24, f"tiny/{d}/{new}")
    lens = [new + 150, new]

    def huge(p):
        p.scale[0] = p.scale[0] * 2.0 ** 119

    paged = Paged(r, lens, 2, 32, d, device, kv=huge)
    rs = starts([new, new])
    q = r.standard_normal((rs[-1], 4, d)) * 2.0 ** -118
    got, lse = attend(paged, rs, lens, q, 4, device)
    check_attention(paged, rs, np.array(lens), q, 4, got, lse)


@pytest.mark.parametrize("d,new", [(128, 1), (64, 1), (128, 6), (64, 20), (128, 60)])
@pytest.mark.parametrize("least", [-60, -20, 0, 30])
def test_pages_of_zeros_beside_values_of_any_size(device, d, new, least):  # noqa: F811
    """Pages whose values are all 0 (their scale is 0) beside pages of very small and of large values: their tokens count in the
    divisor and hide no other."""
    r = syn.rng(25, f"zeros/{d}/{new}/{least}")
    lens = [new + 150, new + 300]

    def some(p):
        p.scale[1] = p.scale[1] * 2.0 ** (least + 9)
        for b in range(2):
            for pg in p.table[b][[0, 2]]:
                p.codes[1][pg], p.scale[1][pg] = 0, 0.0

    paged = Paged(r, lens, 2, 32, d, device, kv=some)
    rs = starts([new, new])
    q = r.standard_normal((rs[-1], 4, d)) * 2.0
    got, lse = attend(paged, rs, lens, q, 4, device)
    check_attention(paged, rs, np.array(lens), q, 4, got, lse)


@pytest.mark.parametrize("d,page", [(128, 64), (64, 16)])
def test_rows_before_the_first_position_are_not_stored(device, d, page):  # noqa: F811
    """An idle slot of length 0 with a row, a sequence shorter than its rows, and an ordinary one: rows at negative positions
    leave the cache as it was, and their queries are rotated all the same."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(26, f"negative/{d}/{page}")
    lens, news, nkv, nh = [0, 2, 40, 0], [1, 5, 3, 2], 2, 4
    paged = Paged(r, lens, nkv, page, d, device)
    rs, T = starts(news), sum(news)
    k, v = (syn.round_bf16(r.standard_normal((T, nkv, d)).astype(np.float32)) for _ in range(2))
    q = syn.round_bf16(r.standard_normal((T, nh, d)).astype(np.float32))
    rope = C.Rope.create(d, 10000.0, device)
    Q = bf16(q.reshape(T, -1), device)
    C.catq_kv_append(paged.cache, i32(rs, device), i32(lens, device), bf16(k.reshape(T, -1), device),
                     bf16(v.reshape(T, -1), device), Q=Q, Q_out=Q, n_heads=nh, rope=rope)
    torch.cuda.synchronize()
    assert C.catq_device_status() == 0
    freq, _ = K.frequencies(d, 10000.0)
    pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, news)])
    want = K.rope(q, pos, freq, False)
    off = np.abs(Q.float().cpu().numpy().reshape(T, nh, d) - want)
    assert (off <= rope_bound(q, freq, False, 1.0) + 2.0 ** -8 * np.abs(want)).all()
    codes, scale = paged.host()
    K.append(paged.codes[1], paged.scale[1], paged.table, page, rs, lens, v.astype(np.float64))
    assert np.array_equal(scale[1], paged.scale[1]) and np.array_equal(K.E4M3[codes[1]], K.E4M3[paged.codes[1]])
    asked = K.append(paged.codes[0], paged.scale[0], paged.table, page, rs, lens, K.rope(k, pos, freq, False))
    kept = np.isnan(asked)
    assert np.array_equal(scale[0], paged.scale[0]) and np.array_equal(K.E4M3[codes[0]][kept], K.E4M3[paged.codes[0]][kept])
    assert kept.sum() == kept.size - 5 * nkv * d  # (2 and 3 tokens are new)


@pytest.mark.parametrize("rows", [1, 2, 3, 9, 30])
def test_heads_of_64_stay_within_the_workspace_of_tiles_of_32_rows(device, rows):
    """Half of the parts' bytes are enough for this call, and what lies behind them is left as it was."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(90, f"half/{rows}")
    lens, news, nh = [9000, 1700], [rows, max(1, rows // 2)], 8
    paged = Paged(r, lens, 2, 64, 64, device)
    T = sum(news)
    q = bf16(r.standard_normal((T, nh * 64)), device)
    args = (paged.cache, i32(starts(news), device), i32(lens, device), q)
    out = [torch.empty(T, nh * 64, dtype=torch.bfloat16, device=device) for _ in range(2)]
    whole = C.kv_attention_workspace(paged.cache, nh)
    half = 4096 + (whole.numel() - 4096) // 2
    C.catq_kv_attention(*args, out[0], nh, whole)
    ws = torch.zeros_like(whole)
    ws[half:] = 77
    C.catq_kv_attention(*args, out[1], nh, ws[:half])
    torch.cuda.synchronize()
    assert C.catq_device_status() == 0
    assert torch.equal(out[0], out[1]) and (ws[half:] == 77).all()
