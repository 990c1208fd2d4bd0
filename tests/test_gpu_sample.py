"""GPU parity of catq_sample with the oracle.  Tokens are the oracle's: weights are whole numbers on both sides, a weight differs
from the oracle's by one at most (2^-44 of its size before it is rounded), and no case draws its u so near a border (the odds
are about V 2^-39 a row).  ln of the probability: two roundings of 64-bit sums to fp32, a division and a logarithm, 2^-21."""
import numpy as np
import pytest

from oracle import tree_oracle as O
from paper_2606_26650_gb300 import synthetic as syn
from tests.test_gpu_kv import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def device():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    return torch.device("cuda:0")


def logits(r, R, V, kind):
    x = r.standard_normal((R, V))
    if kind == "lm":
        x = 2.2 * x + np.where(r.random((R, V)) < 30 / V, r.uniform(4, 15, (R, V)), 0)
    elif kind == "flat":
        x = 1.5 * x
    elif kind == "ties":
        x = np.round(2 * x)
    elif kind == "equal":
        x = np.zeros((R, V)) + 3.5
    elif kind == "few":
        x = np.where(r.random((R, V)) < 5 / V, x, -np.inf)
        x[:, V // 3] = 0.5
    elif kind == "rising":
        x = np.sort(3 * x, axis=1)
    elif kind == "zeros":
        x = np.where(r.random((R, V)) < 0.5, -0.0, 0.0)
        x[:, ::7] = -1e-30
    elif kind == "wide":
        x = 3e38 * np.tanh(x)
    return x


def run(device, x, dtype="f32", gap=0, **kw):
    import torch

    from paper_2606_26650_gb300 import catq as C
    x = np.asarray(x, np.float32)
    R, V = x.shape
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    whole = torch.full((R, V + gap), float("nan"), dtype=dt, device=device)
    X = whole[:, :V]
    X.copy_(torch.from_numpy(x).to(device))
    tokens = torch.full((R + 1,), 77, dtype=torch.int32, device=device)
    lp = torch.full((R + 1,), 77.0, device=device)
    on = {k: None if v is None else (i32(v, device) if k == "top_k" else
                                     torch.tensor(np.asarray(v, np.float32), device=device)) for k, v in kw.items()}
    C.catq_sample(X, on.pop("u"), tokens[:R], logprob=lp[:R], **on)
    torch.cuda.synchronize()
    assert C.catq_device_status() == 0
    assert tokens[R] == 77 and lp[R] == 77
    return X.float().cpu().numpy(), tokens[:R].cpu().numpy(), lp[:R].cpu().numpy()


def check(device, x, dtype="f32", gap=0, **kw):
    read, tokens, lp = run(device, x, dtype, gap, **kw)
    for r in range(len(read)):
        one = {k: np.float32(v[r]) if k != "top_k" else int(v[r]) for k, v in kw.items() if v is not None}
        want, ln = O.sample(read[r], **one)
        assert tokens[r] == want, (r, tokens[r], want, one)
        assert np.isnan(lp[r]) and np.isnan(ln) or abs(lp[r] - ln) <= 2.0 ** -21 * (1e-6 + abs(ln)), (r, lp[r], ln)


def settings(r, R):
    return dict(temperature=np.where(r.random(R) < 0.15, 0, r.uniform(0.3, 1.5, R)),
                top_k=r.choice([0, 1, 2, 20, 1000, 10 ** 6], R), top_p=r.choice([0.0, 0.3, 0.9, 0.95, 1.0], R),
                min_p=r.choice([0.0, 0.0, 0.02, 0.3, 1.0], R))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["lm", "flat", "ties", "equal", "few", "rising", "zeros"])
@pytest.mark.parametrize("R,V,gap", [(1, 1, 0), (3, 2, 1), (4, 7, 0), (5, 33, 3), (9, 1000, 0), (6, 4099, 5), (3, 50001, 0)])
def test_tokens_match_oracle(device, dtype, kind, R, V, gap):
    r = syn.rng(60, f"sample/{kind}/{R}/{V}")
    x = logits(r, R, V, kind)
    check(device, x, dtype, gap, u=r.random(R))
    check(device, x, dtype, gap, u=r.random(R), **settings(r, R))
    for name, value in settings(r, R).items():
        check(device, x, dtype, gap, u=r.random(R), **{name: value})


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_of_many_settings(device, dtype):
    r = syn.rng(61, "many")
    for kind, R, V in (("lm", 300, 700), ("flat", 40, 9000), ("ties", 200, 300), ("lm", 20, 32000)):
        check(device, logits(r, R, V, kind), dtype, 1, u=r.random(R), **settings(r, R))


def test_borders(device):
    """u at both ends, running sums that meet p and u exactly, p of the first token alone."""
    x = np.zeros((8, 16))
    u = np.array([0.0, 1 / 16, 0.5, 15 / 16, 1 - 2.0 ** -24, 1.0, 2.0, -1.0])
    check(device, x, u=u)
    assert run(device, x, u=u)[1].tolist() == [0, 1, 8, 15, 15, 15, 15, 0]
    p = np.array([1 / 16, 0.5, 0.5 + 2.0 ** -20, 1e-30, -1.0, 15 / 16, 1 - 2.0 ** -24, 1.0])
    check(device, x, u=np.full(8, 1 - 2.0 ** -24), top_p=p)
    assert run(device, x, u=np.full(8, 0.9999999), top_p=p)[1].tolist() == [0, 7, 8, 0, 0, 14, 15, 15]
    nan = np.full(8, np.nan)
    check(device, x, u=np.full(8, 0.7), top_p=np.ones(8), min_p=np.zeros(8))
    assert run(device, x, u=np.full(8, 0.7), top_p=nan, min_p=nan)[1].tolist() == [11] * 8
    assert run(device, x, u=nan)[1].tolist() == [0] * 8


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [999, 5000])
def test_temperatures(device, dtype, V):
    r = syn.rng(62, "temperature")
    T = np.array([0.0, 2.0 ** -70, 1e-9, 1e-3, 0.1, 1.0, 30.0, 1e6, 1e30, np.inf])
    for kind in ("lm", "wide", "few"):
        check(device, logits(r, 10, V, kind), dtype, u=r.random(10), temperature=T)
        check(device, logits(r, 10, V, kind), dtype, u=r.random(10), temperature=T, top_p=np.full(10, 0.8), top_k=np.full(10, 300))


def test_temperatures_near_the_limits(device):
    r = syn.rng(62, "temperature")
    check(device, logits(r, 10, 999, "wide"), u=r.random(10), temperature=np.full(10, 3e37))
    # nearby logits at a temperature that tells them apart
    x = 20.0 + np.arange(64)[None] * 2.0 ** -19
    check(device, np.repeat(x, 10, 0), u=r.random(10), temperature=np.full(10, 2.0 ** -15))


def test_rows_from_which_nothing_can_be_drawn(device):
    r = syn.rng(63, "bad")
    for V in (5, 1000, 20000):
        x = logits(r, 7, V, "lm")
        x[0] = -np.inf
        x[1, V - 1] = np.nan
        x[2, 0] = np.inf
        x[3, V // 2] = -np.nan
        t = np.ones(7)
        t[4], t[5] = -1.0, np.nan
        for dtype in ("f32", "bf16"):
            _, tokens, lp = run(device, x, dtype, u=r.random(7), temperature=t)
            assert (tokens[:6] == -1).all() and np.isnan(lp[:6]).all() and tokens[6] >= 0 and lp[6] <= 0
            check(device, x, dtype, u=r.random(7), temperature=t)


def test_frequencies(device):
    """Drawn with evenly spread u, each token comes as often as its probability says, within one."""
    R = 4096
    p = np.array([0.35, 0.05, 0.3, 0.2, 0.1])
    x = np.repeat(np.log(p)[None], R, 0)
    _, tokens, _ = run(device, x, u=(np.arange(R) + 0.5) / R)
    assert np.abs(np.bincount(tokens, minlength=5) - R * p).max() <= 1
    _, tokens, _ = run(device, x, u=(np.arange(R) + 0.5) / R, top_k=np.full(R, 3))
    assert np.abs(np.bincount(tokens, minlength=5) - R * np.array([0.35, 0, 0.3, 0.2, 0]) / 0.85).max() <= 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_vocabularies(device, dtype):
    """More tokens than 16-bit counts hold, all with one logit, and undecided rows of them."""
    r = syn.rng(65, "large")
    V = 600001
    check(device, logits(r, 2, V, "flat"), dtype, 3, u=r.random(2))
    check(device, logits(r, 2, V, "equal"), dtype, 3, u=r.random(2), top_k=np.array([0, 599000]))
    check(device, logits(r, 1, V, "ties"), dtype, 0, u=r.random(1), top_p=np.array([0.7]), min_p=np.array([1e-4]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R", [70, 3000, 70000])
def test_many_rows_that_need_every_logit(device, dtype, R):
    """Rows of 600 equal logits: u of the way through them, each row its own."""
    u = syn.rng(66, "equal").random(R).astype(np.float32)
    _, tokens, lp = run(device, np.full((R, 600), -7.0), dtype, 1, u=u)
    assert np.array_equal(tokens, np.floor(u.astype(np.float64) * 600).astype(np.int64))
    assert np.abs(lp + np.log(600)).max() <= 2.0 ** -21 * np.log(600)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 40, 513, 2048])
def test_rows_that_are_taken_whole(device, dtype, V):
    """Rows without a pass for a bound: no token is lost between a block's first threads and its others, in any call."""
    u = syn.rng(68, "whole").random(20000).astype(np.float32)
    want = np.floor(u.astype(np.float64) * V).astype(np.int64)
    for _ in range(4):
        assert np.array_equal(run(device, np.full((20000, V), 3.0), dtype, 1, u=u)[1], want)


def test_calls_at_once(device):
    """Two streams' calls, which share nothing, give what they give one after the other."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(67, "two")
    x = [torch.tensor(logits(r, 40, 20000, kind), dtype=torch.bfloat16, device=device) for kind in ("lm", "flat")]
    u = torch.tensor(r.random(40), dtype=torch.float32, device=device)
    p = torch.full((40,), 0.95, device=device)
    want = [torch.empty(40, dtype=torch.int32, device=device) for _ in x]
    got = [torch.empty(40, dtype=torch.int32, device=device) for _ in x]
    for a, b in zip(x, want):
        C.catq_sample(a, u, b, top_p=p)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    for _ in range(20):
        for a, b, st in zip(x, got, streams):
            C.catq_sample(a, u, b, top_p=p, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_streams_graphs_and_repeats(device):
    """The same bits each time, on another stream, and replayed with new numbers."""
    import torch

    from paper_2606_26650_gb300 import catq as C
    r = syn.rng(64, "graph")
    R, V = 33, 30000
    x = torch.tensor(logits(r, R, V, "flat"), dtype=torch.bfloat16, device=device)
    u = torch.tensor(r.random(R), dtype=torch.float32, device=device)
    p = torch.full((R,), 0.9, device=device)
    out = [torch.empty(R, dtype=torch.int32, device=device) for _ in range(3)]
    C.catq_sample(x, u, out[0], top_p=p)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    C.catq_sample(x, u, out[1], top_p=p, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(out[0], out[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.catq_sample(x, u, out[2], top_p=p)
    for _ in range(3):
        u.copy_(torch.tensor(r.random(R), dtype=torch.float32))
        graph.replay()
        C.catq_sample(x, u, out[0], top_p=p)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[2])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["flat", "ties", "equal", "rising"])
@pytest.mark.parametrize("R,V,gap", [(64, 12288, 0), (200, 2049, 1), (170, 5003, 0), (63, 4096, 3)])
def test_many_short_rows(device, dtype, kind, R, V, gap):
    r = syn.rng(69, f"short/{kind}/{R}/{V}")
    check(device, logits(r, R, V, kind), dtype, gap, u=r.random(R), **settings(r, R))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R", [40, 1100, 70000])
def test_many_longer_rows_that_need_every_logit(device, dtype, R):
    """As the 600 equal logits, in rows that a cluster takes each."""
    import torch

    from paper_2606_26650_gb300 import catq as C

    V = 12300
    u = syn.rng(70, "longer").random(R).astype(np.float32)
    x = torch.full((R, V), 2.5, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device=device)
    tokens = torch.full((R,), -9, dtype=torch.int32, device=device)
    C.catq_sample(x, torch.from_numpy(u).to(device), tokens)
    assert np.array_equal(tokens.cpu().numpy(), np.floor(u.astype(np.float64) * V).astype(np.int64))


# In rows whose kept weight Z is only known between limits, Z is taken in their middle, 2^-16 of itself at most from either
# one: ln(w / Z) is off by 2^-16 (1 + 2^-16) beside the roundings named above.
def near(lp, ln):
    return abs(lp - ln) <= 2.0 ** -16 * (1 + 2.0 ** -15) + 2.0 ** -21 * abs(ln)


@pytest.mark.parametrize("base,T", [(4.337e6, 1.0), (5.57e6, 1.0), (6.392e6, 1.0), (7.625e6, 1.0), (-7.625e6, 1.0), (1.21e7, 1.0),
                                    (3.1e7, 1.0), (6.7e7, 4.0), (6.392e4, 2.0 ** -7), (9.1e8, 100.0), (1e3, 1.0)])
@pytest.mark.parametrize("V,ties", [(4096, 508), (4099, 300), (40000, 480)])
def test_logits_far_from_zero(device, V, ties, base, T):
    """Logits of a few units in the last place around a number that is large against T: a product of the number with log2(e) / T
    is rounded by a good part of 1, up or down.  About 300 to 508 tokens share the largest."""
    r = syn.rng(71, f"far/{V}/{ties}")
    top = np.float32(base)
    x = np.full(V, top) - np.spacing(np.abs(top)) * r.integers(1, 9, V).astype(np.float32)
    x[r.permutation(V)[:ties]] = top
    order = np.lexsort((np.arange(V), -x))
    w = np.rint(2.0 ** 40 * np.exp((x[order].astype(np.float64) - float(top)) / T)).astype(np.int64)
    upto, share = np.cumsum(w), w[:ties].sum() / w.sum()
    u = np.concatenate([r.random(24) * share, r.random(8)]).astype(np.float32)
    read, tokens, lp = run(device, np.repeat(x[None], 32, 0), u=u, temperature=np.full(32, T))
    assert np.array_equal(read[0], x)
    for i in range(32):
        at = int(np.searchsorted(upto, int(np.floor(np.float64(u[i]) * np.float64(upto[-1]))), side="right"))
        assert tokens[i] == order[at], (i, u[i], at)
        assert near(lp[i], np.log(w[at] / upto[-1])), (i, lp[i], np.log(w[at] / upto[-1]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [20000, 131072])
def test_a_row_beside_others(device, dtype, V):
    """A row by itself and among 64 and 200: the same token; its probability within what Z may be off by, twice."""
    r = syn.rng(73, f"beside/{V}")
    x = logits(r, 1, V, "lm")
    u = r.random(200).astype(np.float32)
    alone = [run(device, x, dtype, u=u[i:i + 1]) for i in range(12)]
    for R in (64, 200):
        _, tokens, lp = run(device, np.repeat(x, R, 0), dtype, u=u[:R])
        for i, (_, t, p) in enumerate(alone):
            assert tokens[i] == t[0]
            assert abs(lp[i] - p[0]) <= 2.0 ** -15 * (1 + 2.0 ** -15) + 2.0 ** -20 * abs(p[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["flat", "equal", "close"])
@pytest.mark.parametrize("R", [1, 4, 66])
def test_the_largest_vocabulary(device, dtype, kind, R):
    """2^20 logits, by eight CTAs a row, four and one.  close: 400 tokens at the largest, all others one step below, so that
    what is not listed weighs as much as it can."""
    V = 1 << 20
    r = syn.rng(72, f"most/{kind}")
    x = logits(r, 1, V, kind)[0].astype(np.float32)
    if kind == "close":
        x = np.full(V, 1.0 - (2.0 ** -24 if dtype == "f32" else 2.0 ** -8), np.float32)
        x[r.permutation(V)[:400]] = 1.0
    u = np.concatenate([[0.5], r.random(R)])[:R].astype(np.float32)
    if kind == "close":
        u[::2] *= np.float32(400 / V)  # (the listed ones)
    read, tokens, lp = run(device, np.repeat(x[None], R, 0), dtype, u=u)
    x = read[0].astype(np.float64)
    order = np.lexsort((np.arange(V), -x))
    w = np.rint(2.0 ** 40 * np.exp(x[order] - x[order[0]])).astype(np.int64)
    upto = np.cumsum(w)
    for i in range(R):
        at = int(np.searchsorted(upto, int(np.floor(np.float64(u[i]) * np.float64(upto[-1]))), side="right"))
        assert tokens[i] == order[at], (i, u[i], at)
        assert near(lp[i], np.log(w[at] / upto[-1]))
