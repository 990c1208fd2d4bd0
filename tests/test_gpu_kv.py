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
])
def test_attention_matches_oracle(device, d, nh, nkv, page, lens, news):
    r = syn.rng(3, f"kv/{d}/{nh}/{nkv}/{page}/{lens}/{news}")
    paged = Paged(r, lens, nkv, page, d, device)
    rs = starts(news)
    q = r.standard_normal((rs[-1], nh, d)) * 2.0
    got, lse = attend(paged, rs, lens, q, nh, device)
    check_attention(paged, rs, np.array(lens), q, nh, got, lse)
