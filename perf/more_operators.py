"""The operators of a decode step that checks a tree of drafted tokens, as measurable cases.

A small model drafts several continuations of each sequence as a tree; the calibrated model looks at all of
its tokens in one pass, a token is drawn at every one of them, and the longest branch that agrees with what
was drawn is kept.  Beside rotary positions, the append and the packed linears that takes five operators:

  masks    the tree, given by every drafted token's parent, as bits of what each sees, and its positions
  tree     attention of the drafted tokens over the paged 8-bit cache: the whole context, and of the drafted
           tokens themselves those on the way from the root
  sample   a token for each row of logits from a given random number: temperature, top-k, top-p, min-p
  accept   the branch whose tokens are the drawn ones, every sequence's next token and new length
  compact  the kept branch's keys and values moved behind the context, in the caches of many layers at once

Head layouts are those of the decoder shapes in paper_2606_26650_gb300/synthetic.py and of the tests; trees,
lengths, batches and numbers of tokens are generic, odd ones among them.
"""
from __future__ import annotations

import math

import torch

own = False

BF, F32, F64, F8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
I32, I64 = torch.int32, torch.int64
E4M3_MAX = 448.0     # the largest e4m3 number
MIN_EXP = -60        # scales are 2^-60 or more
ONE = 2.0 ** 40      # a row's largest weight in sampling: weights are whole multiples of 2^-40


def listed():
    return [
        # One sequence, one small tree: where latency counts.
        dict(name="masks_one", op="masks", B=1, N=8, hi=900),
        # Large trees of many sequences.
        dict(name="masks_batch", op="masks", B=256, N=127, hi=8192),
        # The smallest check: 8 drafted tokens of one short sequence.
        dict(name="tree_short", op="tree", B=1, lo=137, hi=137, N=8, nh=16, nkv=8, d=128, page=64),
        # The ordinary one: 16 sequences of up to 8192 tokens, trees of up to 24.
        dict(name="tree_batch", op="tree", B=16, lo=1000, hi=8192, N=24, nh=32, nkv=8, d=128, page=64),
        # Wide trees, heads of 64 in small pages, few heads a key/value head.
        dict(name="tree_wide_d64", op="tree", B=32, lo=300, hi=4001, N=61, nh=12, nkv=4, d=64, page=16),
        # One row of a small vocabulary: the smallest call.
        dict(name="sample_one", op="sample", R=1, V=32000, dtype="bf16", kind="lm", filters="mixed", gap=0),
        # A decode step of 64 requests, each with settings of its own.
        dict(name="sample_batch", op="sample", R=64, V=131072, dtype="bf16", kind="lm", filters="mixed", gap=0),
        # All rows of a check, 32 bits, an odd vocabulary, plain temperature.
        dict(name="sample_tree_f32", op="sample", R=384, V=100003, dtype="f32", kind="lm", filters="none", gap=5),
        dict(name="accept_one", op="accept", B=1, N=8, hi=900),
        dict(name="accept_batch", op="accept", B=256, N=127, hi=8192),
        # One layer of one sequence.
        dict(name="compact_one", op="compact", L=1, B=1, lo=90, hi=90, N=8, keep=4, nkv=8, d=128, page=64),
        # Sixteen layers of 64 sequences at once, trees that begin and end inside small pages.
        dict(name="compact_layers", op="compact", L=16, B=64, lo=70, hi=150, N=29, keep=9, nkv=8, d=128, page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["masks", "tree", "tree", "sample", "sample", "sample", "accept", "compact"])
    if op in ("masks", "accept"):
        return dict(op=op, B=_log_int(rng, 1, 256), N=_log_int(rng, 1, 127), hi=_log_int(rng, 200, 131072))
    if op == "sample":
        V = _log_int(rng, 1000, 160000)
        R = _log_int(rng, 1, max(1, min(512, 38000000 // V)))
        return dict(op=op, R=R, V=V, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    kind=rng.choice(["lm", "lm", "flat", "allowed"]), filters=rng.choice(["mixed", "mixed", "none"]),
                    gap=rng.choice([0, 0, 1, 24]))
    d = rng.choice([64, 128, 128])
    nkv = rng.choice([1, 2, 4, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "compact":
        N = _log_int(rng, 3, 64)
        hi = N + _log_int(rng, 1, 150)
        return dict(op=op, L=rng.choice([1, 2, 5, 8]), B=_log_int(rng, 1, 64), lo=max(N, hi // rng.choice([1, 2])), hi=hi,
                    N=N, keep=1 + _log_int(rng, 2, N) // 2, nkv=nkv, d=d, page=page)
    nh = nkv * rng.choice([1, 2, 3, 4, 5, 8])
    N = _log_int(rng, 2, 127)
    B = _log_int(rng, 1, 64)
    hi = N + _log_int(rng, 1, min(65536, 500000 // B))
    N = max(1, min(N, 4096 // B, 128000000 // (B * hi * nh) or 1))
    return dict(op=op, B=B, lo=max(N, hi // rng.choice([1, 2, 10])), hi=hi, N=N, nh=nh, nkv=nkv, d=d, page=page)


# ------------------------------------------------------------------ lengths and trees

def _spans(case):
    """Every sequence's length with its drafted tokens, and how many these are."""
    hi, most = case["hi"], case["N"]
    lo = case.get("lo", most)
    lens, news = [], []
    for b in range(case["B"]):
        u, w = ((b + 1) * 0.6180339887) % 1.0, ((b + 1) * 0.4142135623) % 1.0
        news.append(most if b == 0 else 1 + int((most - 1) * w + 0.5))
        lens.append(max(hi if b == 0 else lo + int((hi - lo) * u), news[-1]))
    return lens, news


def _starts(news, dev):
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return torch.tensor(starts, dtype=I32, device=dev)


def _place(row_start, T):
    """Every row's sequence and its place among the sequence's rows."""
    r = torch.arange(T, device=row_start.device)
    b = torch.searchsorted(row_start.long(), r, right=True) - 1
    return b, r - row_start.long()[b]


def _padded(x, row_start, N, fill):
    """[T] as [B, N], `fill` behind a sequence's rows."""
    at = row_start.long()[:-1, None] + torch.arange(N, device=x.device)[None, :]
    return torch.where(at < row_start.long()[1:, None], x[at.clamp(max=max(x.shape[0] - 1, 0))], fill)


def _reach(parent, row_start, N):
    """[B, N, N]: whether j is i or one of its ancestors; parents come before their children."""
    p = _padded(parent.long(), row_start, N, -1)
    j = torch.arange(N, device=p.device)
    m = ((p[:, :, None] == j) | (j[:, None] == j[None, :])).to(F32)
    for _ in range(max(N - 1, 1).bit_length()):  # paths of up to 1, 2, 4 ... steps
        m = torch.matmul(m, m).clamp(max=1.0)
    return m > 0.5


def _packed(bits, words):
    """[..., 32 words] truth values as [..., words] int32, the first in the lowest bit."""
    v = (bits.unflatten(-1, (words, 32)).to(I64) << torch.arange(32, device=bits.device)).sum(dim=-1)
    return torch.where(v >= 2 ** 31, v - 2 ** 32, v).to(I32)


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    s = {"case": dict(case)}

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=dev, dtype=F32)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=F32)

    if case["op"] == "sample":
        R, V = case["R"], case["V"]
        dt = BF if case["dtype"] == "bf16" else F32
        x = normal(R, V + case["gap"])
        if case["kind"] == "flat":        # an undecided model
            x *= 1.5
        else:                             # few tokens stand far above the others, more so in some rows
            x *= 2.2
            x += torch.where(uniform(R, V + case["gap"]) < 30.0 / V, 4.0 + 11.0 * uniform(R, V + case["gap"]), 0.0)
        if case["kind"] == "allowed":     # a grammar leaves some 200 tokens
            x = torch.where(uniform(R, V + case["gap"]) < 200.0 / V, x, -math.inf)
            x[:, V // 2] = 1.0
        s["logits"] = x.to(dt)[:, :V]
        del x
        s["u"] = uniform(R)
        s["temperature"] = s["top_k"] = s["top_p"] = s["min_p"] = None
        if case["filters"] == "mixed":
            def pick(*values):
                i = (uniform(R) * len(values)).long().clamp(max=len(values) - 1)
                return torch.tensor(values, dtype=F32, device=dev)[i]
            s["temperature"] = torch.where(uniform(R) < 0.1, 0.0, 0.5 + 0.7 * uniform(R))
            s["top_k"] = pick(0, 0, 20, 50, 1000).to(I32)
            s["top_p"] = pick(1.0, 0.5, 0.9, 0.95)
            s["min_p"] = pick(0.0, 0.0, 0.05)
        s["tokens"] = torch.empty(R, dtype=I32, device=dev)
        s["logprob"] = torch.empty(R, dtype=F32, device=dev)
        return s

    lens, news = _spans(case)
    B, N, T = case["B"], case["N"], sum(news)
    s["row_start"], s["seq_len"] = _starts(news, dev), torch.tensor(lens, dtype=I32, device=dev)
    _, i = _place(s["row_start"], T)
    # a tree: the first row its root, every other row the child of one of the eight before it
    back = 1 + (uniform(T) * torch.clamp(i, max=8)).long()
    s["parent"] = torch.where(i > 0, (i - back).clamp(min=0), -1).to(I32)
    s["words"] = (N + 31) // 32
    if case["op"] == "masks":
        s["seen"] = torch.empty(T, s["words"], dtype=I32, device=dev)
        s["positions"] = torch.empty(T, dtype=I32, device=dev)
        return s
    if case["op"] == "accept":
        s["sampled"] = (uniform(T) * 1000).to(I32)
        b, _ = _place(s["row_start"], T)
        above = s["sampled"][(s["row_start"].long()[b] + s["parent"].long().clamp(min=0))]
        s["drafted"] = torch.where(uniform(T) < 0.6, above, (uniform(T) * 1000).to(I32))
        s["path"] = torch.empty(T, dtype=I32, device=dev)
        s["kept"], s["next"], s["new_len"] = (torch.empty(B, dtype=I32, device=dev) for _ in range(3))
        return s

    nkv, d, page, L = case["nkv"], case["d"], case["page"], case.get("L", 1)
    need = [-(-n // page) for n in lens]
    width, total = max(need), sum(need)
    n_pages = total + 3
    order = torch.randperm(n_pages, generator=g, device=dev)[:total].cpu()
    table = torch.full((B, width), -1, dtype=I32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = table.to(dev)
    loud = 1.0 + 4.0 * (uniform(nkv, 1, d) < 0.03)  # a few loud channels of the keys
    for n, gain in (("k", loud), ("v", 1.0)):
        x = normal(L, n_pages, nkv, page, d) * gain
        x *= torch.exp2(torch.floor(3.0 * uniform(L, n_pages, nkv, 1, 1)))  # pages of unlike magnitude
        scale = _scale_of(x.abs().amax(dim=(3, 4)))
        s[n + "_codes"], s[n + "_scale"] = (x / scale[..., None, None]).to(F8), scale
        del x
    if case["op"] == "compact":
        # branches of up to `keep` rows: the root, and rows that lie behind the kept ones' new places
        kept, path = [], torch.full((T,), -1, dtype=I32)
        shuffled, at = uniform(T).cpu().tolist(), 0
        for b, n in enumerate(news):
            m = max(1, min(case["keep"], (n + 1) // 2) - b % 3)
            rest = sorted(sorted(range(m, n), key=lambda j: shuffled[at + j])[:m - 1])
            path[at:at + 1 + len(rest)] = torch.tensor([0] + rest, dtype=I32)
            kept.append(1 + len(rest))
            at += n
        s["path"], s["kept"] = path.to(dev), torch.tensor(kept, dtype=I32, device=dev)
        return s
    for n in ("k", "v"):
        s[n + "_codes"], s[n + "_scale"] = s[n + "_codes"][0], s[n + "_scale"][0]
    s["seen"] = _packed(torch.nn.functional.pad(_reach(s["parent"], s["row_start"], N), (0, 32 * s["words"] - N)),
                        s["words"])[_place(s["row_start"], T)]
    s["q"] = (normal(T, case["nh"] * d) * 1.5).to(BF)
    s["o"] = torch.zeros_like(s["q"])
    return s


def _scale_of(top):
    """The least power of two (2^MIN_EXP at least) that brings values up to `top` to 448 or below; 0 for 0."""
    f, e = torch.frexp(top)  # top = f 2^e, 1/2 <= f < 1; 448 = 7/8 2^9
    k = torch.where(f <= 0.875, e - 9, e - 8).clamp(min=MIN_EXP)
    return torch.where(top > 0, torch.ldexp(torch.ones_like(top), k), torch.zeros_like(top))


# ------------------------------------------------------------------ one pass

def run(state):
    op = state["case"]["op"]
    if own:
        return {"masks": _own_masks, "tree": _own_tree, "sample": _own_sample, "accept": _own_accept,
                "compact": _own_compact}[op](state)
    return {"masks": _plain_masks, "tree": _plain_tree, "sample": _plain_sample, "accept": _plain_accept,
            "compact": _plain_compact}[op](state)


def _own_masks(s):
    from paper_2606_26650_gb300 import catq as C
    C.catq_tree_masks(s["parent"], s["row_start"], s["seq_len"], s["seen"], s["positions"])
    return {"seen": s["seen"], "positions": s["positions"]}


def _own_tree(s):
    from paper_2606_26650_gb300 import catq as C
    c = s["case"]
    if "cache" not in s:
        s["cache"] = C.KVCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["table"])
        s["workspace"] = C.kv_attention_workspace(s["cache"], c["nh"])
    C.catq_kv_tree_attention(s["cache"], s["row_start"], s["seq_len"], s["seen"], s["q"], s["o"], c["nh"],
                             s["workspace"])
    return s["o"]


def _own_sample(s):
    from paper_2606_26650_gb300 import catq as C
    C.catq_sample(s["logits"], s["u"], s["tokens"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                  min_p=s["min_p"], logprob=s["logprob"])
    return {"tokens": s["tokens"], "logprob": s["logprob"]}


def _own_accept(s):
    from paper_2606_26650_gb300 import catq as C
    C.catq_tree_accept(s["drafted"], s["sampled"], s["parent"], s["row_start"], s["seq_len"], s["path"], s["kept"],
                       s["next"], s["new_len"])
    return {"path": s["path"], "kept": s["kept"], "next": s["next"], "new_len": s["new_len"]}


def _own_compact(s):
    from paper_2606_26650_gb300 import catq as C
    if "caches" not in s:
        s["caches"] = [C.KVCache(*(s[n][i] for n in ("k_codes", "v_codes", "k_scale", "v_scale")), s["table"])
                       for i in range(s["case"]["L"])]
    C.catq_kv_compact(s["caches"], s["row_start"], s["seq_len"], s["path"], s["kept"])
    return {"k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ------------------------------------------------------------------ the plain forms

def _plain_masks(s):
    N, T, words = s["case"]["N"], s["parent"].shape[0], s["words"]
    m = _reach(s["parent"], s["row_start"], N)
    b, i = _place(s["row_start"], T)
    s["seen"].copy_(_packed(torch.nn.functional.pad(m, (0, 32 * words - N)), words)[b, i])
    first = s["seq_len"].long() - (s["row_start"][1:] - s["row_start"][:-1]).long()
    s["positions"].copy_(first[b] + m.sum(dim=-1)[b, i] - 1)
    return {"seen": s["seen"], "positions": s["positions"]}


def _plain_tree(s):
    c = s["case"]
    B, nh, nkv, d, page, N = c["B"], c["nh"], c["nkv"], c["d"], c["page"], c["N"]
    T = s["q"].shape[0]
    pages = s["table"].long().clamp(min=0)
    L = pages.shape[1] * page

    def cached(n):  # [B, nkv, L, d]
        x = s[n + "_codes"].view(torch.uint8)[pages].view(F8).to(F32) * s[n + "_scale"][pages][..., None, None]
        return x.transpose(1, 2).reshape(B, nkv, L, d)

    start = s["row_start"].long()
    new = start[1:] - start[:-1]
    i = torch.arange(N, device=start.device)
    rows = (start[:-1, None] + i[None, :]).clamp(max=T - 1)
    q = s["q"].to(F32).view(T, nkv, nh // nkv, d)[rows]            # [B, N, nkv, group, d]
    q = q.permute(0, 2, 3, 1, 4).reshape(B, nkv, (nh // nkv) * N, d)
    score = torch.matmul(q, cached("k").transpose(2, 3)) / math.sqrt(d)
    # a place of the cache is one of the context, or the j-th drafted token, which a row sees by its bit j
    j = torch.arange(L, device=start.device)[None, :] - (s["seq_len"].long() - new)[:, None]
    bits = (s["seen"][rows][..., None].long() >> torch.arange(32, device=start.device)) & 1     # [B, N, words, 32]
    bits = bits.flatten(2).gather(2, j.clamp(0, 32 * s["words"] - 1)[:, None, :].expand(-1, N, -1)) > 0
    seen = (j < 0)[:, None] | (bits & (j < new[:, None])[:, None])
    score = score.view(B, nkv, nh // nkv, N, L).masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(score - score.amax(dim=-1, keepdim=True).clamp(min=-3e38))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, nkv, -1, L), cached("v")).view(B, nkv, nh // nkv, N, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    s["o"].copy_(o.permute(0, 3, 1, 2, 4)[_place(s["row_start"], T)].reshape(T, nh * d))
    return s["o"]


def _plain_sample(s):
    x, V = s["logits"], s["case"]["V"]
    R, dev = x.shape[0], x.device

    def setting(n, default):
        return torch.full((R,), default, dtype=F64, device=dev) if s[n] is None else s[n].to(F64)

    temperature = setting("temperature", 1.0)
    greedy = temperature == 0
    wide = x.to(F64)
    by = torch.where(greedy, 1.0, temperature)[:, None]
    weight = (torch.exp((wide - wide.amax(dim=1, keepdim=True)) / by) * ONE).round().to(I64)
    order = torch.sort(x.to(F32), dim=1, descending=True, stable=True).indices
    weight = weight.gather(1, order)
    upto = weight.cumsum(dim=1)
    # every filter leaves a first part of the tokens in falling order
    k = setting("top_k", 0.0).to(I64)
    k = torch.where(greedy, 1, torch.where(k <= 0, V, k.clamp(max=V)))
    whole = upto.gather(1, (k - 1)[:, None])[:, 0]
    p = setting("top_p", 1.0)
    need = torch.where(p < 1, (p * whole.to(F64)).ceil().to(I64).clamp(min=1).minimum(whole), whole)
    least = (setting("min_p", 0.0) * ONE).ceil().clamp(1.0, ONE).to(I64)
    kept = torch.minimum(torch.minimum(k, (upto < need[:, None]).sum(dim=1) + 1),
                         (weight >= least[:, None]).sum(dim=1))
    total = upto.gather(1, (kept - 1)[:, None])[:, 0]
    at = (s["u"].to(F64) * total.to(F64)).floor().to(I64).clamp(min=0).minimum(total - 1)
    place = (upto <= at[:, None]).sum(dim=1, keepdim=True)
    s["tokens"].copy_(order.gather(1, place)[:, 0])
    s["logprob"].copy_(torch.log(weight.gather(1, place)[:, 0].to(F64) / total.to(F64)))
    return {"tokens": s["tokens"], "logprob": s["logprob"]}


def _plain_accept(s):
    c = s["case"]
    N, T, dev = c["N"], s["parent"].shape[0], s["parent"].device
    start = s["row_start"].long()
    new = start[1:] - start[:-1]
    parent = _padded(s["parent"].long(), s["row_start"], N, -1)
    drafted, sampled = (_padded(s[n].long(), s["row_start"], N, -1) for n in ("drafted", "sampled"))
    # a row is chosen among its siblings if it is the first whose token was drawn at their parent
    fits = (parent >= 0) & (drafted == sampled.gather(1, parent.clamp(min=0)))
    i = torch.arange(N, device=dev)
    first = torch.full((c["B"], N), N, dtype=I64, device=dev)
    first = first.scatter_reduce(1, parent.clamp(min=0), torch.where(fits, i, N), "amin")
    chosen = fits & (first.gather(1, parent.clamp(min=0)) == i)
    chosen[:, 0] = True
    reach = _reach(s["parent"], s["row_start"], N)
    kept = (reach[:, :, 0] & ~(reach & ~chosen[:, None, :]).any(dim=2)) & (i < new[:, None])
    count = kept.sum(dim=1)
    # the kept rows in their order, then -1
    path = torch.where(kept, i, N).sort(dim=1).values
    b, place = _place(s["row_start"], T)
    s["path"].copy_(torch.where(path < N, path, -1)[b, place])
    s["kept"].copy_(count)
    last = path.gather(1, (count - 1).clamp(min=0)[:, None])
    s["next"].copy_(torch.where(count > 0, sampled.gather(1, last.clamp(max=N - 1))[:, 0], -1))
    s["new_len"].copy_(s["seq_len"].long() - new + count)
    return {"path": s["path"], "kept": s["kept"], "next": s["next"], "new_len": s["new_len"]}


def _plain_compact(s):
    c = s["case"]
    L, nkv, page, T = c["L"], c["nkv"], c["page"], s["path"].shape[0]
    b, j = _place(s["row_start"], T)
    moved = (j < s["kept"].long()[b]) & (s["path"] != j)
    b, j, i = b[moved], j[moved], s["path"].long()[moved]
    first = (s["seq_len"] - (s["row_start"][1:] - s["row_start"][:-1])).long()[b]
    src, dst = first + i, first + j
    src_page, dst_page = s["table"].long()[b, src // page], s["table"].long()[b, dst // page]
    gets = torch.unique(dst_page)                         # pages that get tokens
    for n in ("k", "v"):
        codes, scale = s[n + "_codes"], s[n + "_scale"]
        bytes_ = codes.view(torch.uint8)
        value = (bytes_[:, src_page, :, src % page].view(F8).to(F32)               # [moved, L, nkv, d]
                 * scale[:, src_page].transpose(0, 1)[..., None])
        top = torch.zeros_like(scale).index_reduce_(1, dst_page, value.abs().amax(dim=-1).transpose(0, 1), "amax")
        grown = torch.maximum(scale, _scale_of(top))
        ratio = torch.where(grown > 0, scale / grown, torch.ones_like(grown))[:, gets][..., None, None]
        bytes_[:, gets] = (bytes_[:, gets].view(F8).to(F32) * ratio).to(F8).view(torch.uint8)
        scale.copy_(grown)
        by = scale[:, dst_page].transpose(0, 1)[..., None]
        bytes_[:, dst_page, :, dst % page] = torch.where(by > 0, value / by, value).to(F8).view(torch.uint8)
    return {"k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


# ------------------------------------------------------------------ 64 bits

def _exact_e4m3(x):
    """The nearest e4m3 number, ties to the even one, for |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _ways(parent):
    """Every row's ancestors, itself last, of one tree as a list of parents."""
    out = []
    for i, p in enumerate(parent):
        out.append((out[p] if p >= 0 else []) + [i])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "sample":
        return _exact_sample(s)
    lens, news = _spans(c)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    parents = s["parent"].cpu().tolist()
    trees = [_ways(parents[a:z]) for a, z in zip(starts, starts[1:])]
    if c["op"] == "masks":
        seen, pos = [], []
        for n, k, tree in zip(lens, news, trees):
            for way in tree:
                bits = sum(1 << i for i in way)
                seen.append([((bits >> 32 * w & 0xFFFFFFFF) ^ 0x80000000) - 0x80000000 for w in range(s["words"])])
                pos.append(n - k + len(way) - 1)
        return {"seen": torch.tensor(seen, dtype=I32), "positions": torch.tensor(pos, dtype=I32)}
    if c["op"] == "accept":
        drafted, sampled = s["drafted"].cpu().tolist(), s["sampled"].cpu().tolist()
        out = {"path": [], "kept": [], "next": [], "new_len": []}
        for b, (n, k) in enumerate(zip(lens, news)):
            a, way = starts[b], [0]
            while True:
                more = [i for i in range(1, k) if parents[a + i] == way[-1] and drafted[a + i] == sampled[a + way[-1]]]
                if not more:
                    break
                way.append(more[0])
            out["path"] += way + [-1] * (k - len(way))
            out["kept"].append(len(way))
            out["next"].append(sampled[a + way[-1]])
            out["new_len"].append(n - k + len(way))
        return {n: torch.tensor(v, dtype=I32) for n, v in out.items()}
    table, page, nkv, d = s["table"].cpu().tolist(), c["page"], c["nkv"], c["d"]
    if c["op"] == "compact":
        out = {}
        path, kept = s["path"].cpu().tolist(), s["kept"].cpu().tolist()
        for n in "kv":
            codes, scale = s[n + "_codes"].to(F64), s[n + "_scale"].to(F64)
            for b, (length, k) in enumerate(zip(lens, news)):
                first, way = length - k, path[starts[b]:starts[b] + kept[b]]
                for number in range(first // page, (first + len(way) - 1) // page + 1):
                    # (slot, where its token lies) of what comes into this page
                    moves = [(first + j, first + i) for j, i in enumerate(way)
                             if i != j and (first + j) // page == number]
                    if not moves:
                        continue
                    p = table[b][number]
                    old = torch.stack([codes[:, table[b][i // page], :, i % page] * scale[:, table[b][i // page], :, None]
                                       for _, i in moves], dim=2)                      # [L, nkv, moved, d]
                    part, power = torch.frexp(old.abs().amax(dim=(2, 3)) / E4M3_MAX)
                    want = torch.exp2((power - (part == 0.5).to(power.dtype)).to(F64).clamp(min=MIN_EXP))
                    now = torch.maximum(scale[:, p], torch.where(part > 0, want, 0.0))
                    by = torch.where(now > 0, now, 1.0)
                    codes[:, p] = _exact_e4m3(codes[:, p] * (scale[:, p] / by)[..., None, None])
                    scale[:, p] = now
                    codes[:, p, :, [j % page for j, _ in moves]] = _exact_e4m3(old / by[..., None, None])
            out[n], out[n + "_scale"] = codes, scale
        return {n: out[n] for n in ("k", "v", "k_scale", "v_scale")}
    nh = c["nh"]
    out = torch.zeros(sum(news), nh, d, dtype=F64, device=s["q"].device)
    for b, (n, k) in enumerate(zip(lens, news)):
        pages = torch.tensor(table[b][:-(-n // page)], device=s["q"].device)
        hidden = torch.zeros(k, n, dtype=torch.bool)
        hidden[:, n - k:] = True
        for i, way in enumerate(trees[b]):
            hidden[i, [n - k + j for j in way]] = False
        hidden = hidden.to(s["q"].device)
        for h in range(nkv):
            key, val = ((s[x + "_codes"].view(torch.uint8)[pages, h].view(F8).to(F64)
                         * s[x + "_scale"][pages, h].to(F64)[:, None, None]).reshape(-1, d)[:n] for x in "kv")
            heads = slice(h * (nh // nkv), (h + 1) * (nh // nkv))
            q = s["q"][starts[b]:starts[b] + k].to(F64).view(k, nh, d)[:, heads].transpose(0, 1)
            weight = torch.softmax((q @ key.T * d ** -0.5).masked_fill(hidden, -math.inf), dim=-1)
            out[starts[b]:starts[b] + k, heads] = (weight @ val).transpose(0, 1)
    return out.flatten(1)


def _exact_sample(s):
    """Row by row, by its distinct values: how many tokens have each and what they weigh together."""
    x = s["logits"]
    of = {n: (None if s[n] is None else s[n].cpu().tolist()) for n in ("temperature", "top_k", "top_p", "min_p", "u")}
    tokens, logprob = [], []
    for r in range(x.shape[0]):
        value, count = torch.unique(x[r].to(F64), return_counts=True)
        value, count = value.flip(0), count.flip(0)           # falling
        t = 1.0 if of["temperature"] is None else of["temperature"][r]
        if t == 0.0:
            tokens.append(int((x[r] == value[0]).nonzero()[0, 0]))
            logprob.append(0.0)
            continue
        weight = torch.round(2.0 ** 40 * torch.exp((value - value[0]) / t)).to(I64)
        left = x.shape[1] if of["top_k"] is None or of["top_k"][r] <= 0 else of["top_k"][r]
        count = torch.minimum(count, (left - (count.cumsum(0) - count)).clamp(min=0))
        whole = int((count * weight).sum())
        if of["top_p"] is not None and of["top_p"][r] < 1.0:
            need = min(max(math.ceil(of["top_p"][r] * float(whole)), 1), whole)
            before = (count * weight).cumsum(0) - count * weight
            fit = torch.div(need - before + weight.clamp(min=1) - 1, weight.clamp(min=1), rounding_mode="floor")
            count = torch.minimum(count, fit.clamp(min=0))
        least = 1.0 if of["min_p"] is None else min(max(math.ceil(of["min_p"][r] * 2.0 ** 40), 1.0), 2.0 ** 40)
        count = torch.where(weight >= least, count, 0)
        total = int((count * weight).sum())
        at = min(max(math.floor(of["u"][r] * float(total)), 0), total - 1)
        upto = (count * weight).cumsum(0)
        v = int((upto <= at).sum())
        nth = (at - int(upto[v] - count[v] * weight[v])) // int(weight[v])
        tokens.append(int((x[r].to(F64) == value[v]).nonzero()[nth, 0]))
        logprob.append(math.log(int(weight[v]) / total))
    return {"tokens": torch.tensor(tokens, dtype=I32), "logprob": torch.tensor(logprob, dtype=F64)}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "sample":
        return {"bytes": c["R"] * c["V"] * (2 if c["dtype"] == "bf16" else 4) + 28 * c["R"], "flops": 4 * c["R"] * c["V"]}
    lens, news = _spans(c)
    B, T, words = c["B"], sum(news), (c["N"] + 31) // 32
    if c["op"] == "masks":
        return {"bytes": 4 * T + 8 * B + 4 * T * words + 4 * T, "flops": T}
    if c["op"] == "accept":
        return {"bytes": 4 * 4 * T + 5 * 4 * B, "flops": T}
    nkv, d, page = c["nkv"], c["d"], c["page"]
    if c["op"] == "compact":
        rows = sum(max(1, min(c["keep"], (n + 1) // 2) - b % 3) - 1 for b, n in enumerate(news))
        # the moved tokens' codes read and written, a page's scales read and written
        return {"bytes": c["L"] * 2 * nkv * (2 * rows * d + 2 * 4 * B) + 4 * T, "flops": c["L"] * 2 * nkv * rows * d}
    nh = c["nh"]
    bytes_ = sum(2 * n * nkv * d + 2 * 4 * -(-n // page) * nkv for n in lens) + 2 * T * nh * d * 2 + 4 * T * words
    return {"bytes": bytes_, "flops": sum(4 * nh * d * k * (n - k + 1) for n, k in zip(lens, news))}
