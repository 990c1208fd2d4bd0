"""The operators of the deployed model's decoding, as measurable cases.

A calibrated model is served token by token: its packed linears run through catq_ternary_infer, and
between them every new token's query and key are rotated to the token's position, its key and value go
into a paged cache of 8-bit codes, and its query attends to all that the cache holds of its sequence.
Three operators:

  rope       rotary positions given per token: pairs in halves or interleaved, a part of the head, with
             the frequencies scaled for long contexts; forward, and inverse (the backward)
  append     new keys and values into the paged 8-bit cache: the keys rotated on the way, a power-of-two
             scale for each page and head that grows with the page's values (the codes already there
             follow it), the queries rotated in the same call
  attention  grouped-query attention of the new tokens over the cache, causal among themselves

Head layouts are those of the decoder shapes in paper_2606_26650_gb300/synthetic.py (16 / 8, 32 / 8 and
40 / 8 heads of 128) and of the tests (heads of 64); lengths and batches are generic, odd ones among them.
The cache's elements are e4m3 numbers: codes are returned as the float8 numbers they are, beside their scales.
"""
from __future__ import annotations

import math

import torch

own = False

BF, F32, F64, F8 = torch.bfloat16, torch.float32, torch.float64, torch.float8_e4m3fn
E4M3_MAX = 448.0     # the largest e4m3 number
MIN_EXP = -60        # scales are 2^-60 or more


def listed():
    return [
        # One decode step of 64 sequences at far positions: where latency counts.
        dict(name="rope_token", op="rope", T=64, nh=32, d=128, rot=128, interleaved=False, dtype="bf16", far=131072,
             scaling="bands", inverse=False, gap=2048),
        # A prefill of 4 x 2048 tokens, the queries in the rows of a fused q/k/v product.
        dict(name="rope_prefill", op="rope", T=8192, nh=32, d=128, rot=128, interleaved=False, dtype="bf16", far=8192,
             scaling="bands", inverse=False, gap=2048),
        # The backward of interleaved pairs over half the head, fp32, an odd number of tokens.
        dict(name="rope_backward_f32", op="rope", T=4999, nh=40, d=128, rot=64, interleaved=True, dtype="f32", far=32768,
             scaling="yarn", inverse=True, gap=0),
        # One token for each of 64 sequences of unequal length.
        dict(name="append_token", op="append", B=64, lo=1, hi=700, new=1, nh=32, nkv=8, d=128, page=64, rot=128,
             interleaved=False, scaling="bands"),
        # Whole prompts: 4 x 2048 tokens into empty pages.
        dict(name="append_prompt", op="append", B=4, lo=2048, hi=2048, new=2048, nh=32, nkv=8, d=128, page=64, rot=128,
             interleaved=False, scaling="bands"),
        # Odd chunks that begin and end inside small pages, heads of 64, a quarter of the head rotated.
        dict(name="append_ragged_d64", op="append", B=37, lo=90, hi=611, new=83, nh=12, nkv=4, d=64, page=16, rot=16,
             interleaved=True, scaling="none"),
        # A single short sequence: the smallest call.
        dict(name="attn_short", op="attention", B=1, lo=137, hi=137, new=1, nh=16, nkv=8, d=128, page=64),
        # The ordinary decode step: 64 sequences of up to 8192 tokens.
        dict(name="attn_batch", op="attention", B=64, lo=300, hi=8192, new=1, nh=32, nkv=8, d=128, page=64),
        # One long context.
        dict(name="attn_long", op="attention", B=1, lo=131071, hi=131071, new=1, nh=32, nkv=8, d=128, page=128),
        # Up to five drafted tokens a sequence are checked at once, 5 query heads a key/value head.
        dict(name="attn_draft", op="attention", B=16, lo=1000, hi=4500, new=5, nh=40, nkv=8, d=128, page=32),
        # A prompt's next chunk over what is cached of it.
        dict(name="attn_chunk", op="attention", B=2, lo=6001, hi=8191, new=1023, nh=32, nkv=8, d=128, page=64),
        # Heads of 64 with no sharing, small pages, many sequences.
        dict(name="attn_heads64", op="attention", B=128, lo=17, hi=2001, new=1, nh=12, nkv=12, d=64, page=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention"])
    d = rng.choice([64, 128, 128])
    nkv = rng.choice([1, 2, 4, 8])
    nh = nkv * rng.choice([1, 2, 3, 4, 5, 8])
    if op == "rope":
        T = _log_int(rng, 1, 8192)
        return dict(op=op, T=T, nh=nh, d=d, rot=rng.choice([d, d, d // 2, d // 4]), interleaved=rng.random() < 0.5,
                    dtype=rng.choice(["bf16", "f32"]), far=_log_int(rng, 4096, 131072),
                    scaling=rng.choice(["none", "linear", "bands", "yarn"]), inverse=rng.random() < 0.5,
                    gap=rng.choice([0, 0, 64, 2 * nkv * d]))
    page = rng.choice([16, 32, 64, 128])
    B = _log_int(rng, 1, 128)
    if op == "append":
        new = _log_int(rng, 1, max(1, 8192 // B)) if rng.random() < 0.6 else 1
        hi = new + _log_int(rng, 1, max(2, 40000 // B))
        return dict(op=op, B=B, lo=max(1, hi // rng.choice([1, 2, 5])), hi=hi, new=new, nh=nh, nkv=nkv, d=d, page=page,
                    rot=rng.choice([d, d, d // 2, d // 4]), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "bands", "yarn"]))
    hi = _log_int(rng, 16, min(131072, 500000 // B))
    new = rng.choice([1, 1, 1, 2, 7, _log_int(rng, 8, 1024)])
    new = max(1, min(new, hi, 2048 // B, 128000000 // (B * hi * nh) or 1))
    return dict(op=op, B=B, lo=max(1, hi // rng.choice([1, 2, 10])), hi=hi, new=new, nh=nh, nkv=nkv, d=d, page=page)


# ------------------------------------------------------------------ lengths and frequencies

def _spans(case):
    """Every sequence's tokens in the cache after the call, and how many of them are the call's."""
    lo, hi, most = case["lo"], case["hi"], case["new"]
    lens, news = [], []
    for b in range(case["B"]):
        u, w = ((b + 1) * 0.6180339887) % 1.0, ((b + 1) * 0.4142135623) % 1.0
        n = hi if b == 0 else lo + int((hi - lo) * u)
        k = most if b == 0 or lo == hi else 1 + int((most - 1) * w + 0.5)
        lens.append(n)
        news.append(min(k, n))
    return lens, news


def _frequencies(rot, scaling, base=500000.0):
    """Radians a token of each pair (64 bits), and the factor on the rotated values: as they are, all
    slowed down (positions interpolated by 8), by wavelength in three bands, or by a ramp over the turns
    that a pair makes in the original context (with the scores' temperature)."""
    i = torch.arange(0, rot, 2, dtype=F64)
    f = base ** (-i / rot)
    factor, original = 8.0, 8192.0
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "bands":
        low, high = 1.0, 4.0
        turns = original * f / (2 * math.pi)
        mix = ((turns - low) / (high - low)).clamp(0.0, 1.0)
        return (1 - mix) * f / factor + mix * f, 1.0
    if scaling == "yarn":
        fast, slow = 32.0, 1.0

        def dim(turns):
            return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))

        a, b = max(math.floor(dim(fast)), 0), min(math.ceil(dim(slow)), rot - 1)
        ramp = ((torch.arange(rot // 2, dtype=F64) - a) / max(b - a, 0.001)).clamp(0.0, 1.0)
        return ramp * f / factor + (1 - ramp) * f, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _turns(freq):
    """Turns a token as 64-bit fixed point: 2^64 is one turn."""
    return (freq / (2 * math.pi) * 2.0 ** 62).round().to(torch.int64) * 4


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=F32)

    s = {"case": dict(case)}
    if case["op"] != "attention":
        freq, magnitude = _frequencies(case["rot"], case["scaling"])
        s["freq"], s["turns"], s["magnitude"] = freq.to(dev), _turns(freq).to(dev), magnitude
    if case["op"] == "rope":
        T, width, dt = case["T"], case["nh"] * case["d"], BF if case["dtype"] == "bf16" else F32
        s["x"] = normal(T, width + case["gap"]).to(dt)[:, :width]
        s["y"] = torch.empty(T, width, dtype=dt, device=dev)
        s["pos"] = torch.randint(0, case["far"], (T,), generator=g, device=dev, dtype=torch.int32)
        return s
    nh, nkv, d, page, B = case["nh"], case["nkv"], case["d"], case["page"], case["B"]
    lens, news = _spans(case)
    need = [-(-n // page) for n in lens]
    width, total = max(need), sum(need)
    n_pages = total + 3
    order = torch.randperm(n_pages, generator=g, device=dev)[:total].cpu()
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"] = table.to(dev)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device=dev)
    s["seq_len"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    s["max_len"], s["max_new"] = max(lens), max(news)
    T = starts[-1]
    loud = 1.0 + 4.0 * (torch.rand(nkv, 1, d, generator=g, device=dev) < 0.03)  # a few loud channels of the keys
    for n, gain in (("k", loud), ("v", 1.0)):
        x = normal(n_pages, nkv, page, d) * gain
        scale = _scale_of(x.abs().amax(dim=(2, 3)))
        s[n + "_codes"], s[n + "_scale"] = (x / scale[..., None, None]).to(F8), scale
        del x
    s["q"] = (normal(T, nh * d) * 1.5).to(BF)
    if case["op"] == "append":
        s["q_out"] = torch.empty_like(s["q"])
        rows = normal(T, 2, nkv, d)
        rows[:, 0] *= loud.transpose(0, 1)
        # values a little larger than the cached ones in some rows, so that scales grow
        rows *= 1.0 + (torch.rand(T, 1, 1, 1, generator=g, device=dev) < 0.1)
        fused = rows.to(BF).view(T, 2 * nkv * d)
        s["k"], s["v"] = fused[:, :nkv * d], fused[:, nkv * d:]
    else:
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
        return {"rope": _own_rope, "append": _own_append, "attention": _own_attention}[op](state)
    return {"rope": _plain_rope, "append": _plain_append, "attention": _plain_attention}[op](state)


def _rope_handle(s):
    from paper_2606_26650_gb300 import catq as C
    if "rope" not in s:
        c = s["case"]
        s["rope"] = C.Rope(s["turns"], c["rot"], C.ROPE_INTERLEAVED if c["interleaved"] else C.ROPE_HALF, s["magnitude"])
    return C, s["rope"]


def _cache_handle(s):
    from paper_2606_26650_gb300 import catq as C
    if "cache" not in s:
        s["cache"] = C.KVCache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["table"])
    return C, s["cache"]


def _own_rope(s):
    C, rope = _rope_handle(s)
    c = s["case"]
    C.catq_rope_at(s["x"], s["pos"], rope, c["nh"], c["d"], s["y"], inverse=c["inverse"])
    return s["y"]


def _own_append(s):
    _, rope = _rope_handle(s)
    C, cache = _cache_handle(s)
    C.catq_kv_append(cache, s["row_start"], s["seq_len"], s["k"], s["v"], rope=rope, Q=s["q"], Q_out=s["q_out"],
                     n_heads=s["case"]["nh"])
    return {"k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "q": s["q_out"]}


def _own_attention(s):
    C, cache = _cache_handle(s)
    c = s["case"]
    if "workspace" not in s:
        s["workspace"] = C.kv_attention_workspace(cache, c["nh"])
    C.catq_kv_attention(cache, s["row_start"], s["seq_len"], s["q"], s["o"], c["nh"], s["workspace"])
    return s["o"]


# ------------------------------------------------------------------ the plain forms

def _plain_rotate(x, pos, s, inverse=False):
    """x [T, heads, d] (fp32) with the first `rot` elements of every head rotated: angles in 64 bits."""
    c = s["case"]
    rot = c["rot"]
    angle = pos.to(F64)[:, None] * s["freq"][None, :]
    cos, sin = (angle.cos() * s["magnitude"]).to(F32)[:, None, :], (angle.sin() * s["magnitude"]).to(F32)[:, None, :]
    if inverse:
        sin = -sin
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :rot // 2], r[..., rot // 2:])
    p, q = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((p, q), dim=-1).flatten(-2) if c["interleaved"] else torch.cat((p, q), dim=-1)
    return torch.cat((r, x[..., rot:]), dim=-1)


def _plain_rope(s):
    c = s["case"]
    x = s["x"].to(F32).view(c["T"], c["nh"], c["d"])
    s["y"].copy_(_plain_rotate(x, s["pos"], s, c["inverse"]).view(c["T"], -1))
    return s["y"]


def _rows_of(s, T):
    """Sequence, place among the sequence's new tokens and position of every row."""
    r = torch.arange(T, device=s["q"].device)
    b = torch.searchsorted(s["row_start"].long(), r, right=True) - 1
    i = r - s["row_start"].long()[b]
    new = (s["row_start"][1:] - s["row_start"][:-1]).long()
    return b, i, s["seq_len"].long()[b] - new[b] + i


def _plain_append(s):
    c = s["case"]
    nkv, d, page = c["nkv"], c["d"], c["page"]
    T = s["q"].shape[0]
    b, _, pos = _rows_of(s, T)
    s["q_out"].copy_(_plain_rotate(s["q"].to(F32).view(T, c["nh"], d), pos, s).view(T, -1))
    blocks = s["table"].long()[b, pos // page]                     # the page of every row
    first = (s["seq_len"] - (s["row_start"][1:] - s["row_start"][:-1])).long()  # each sequence's first new position
    seq = torch.arange(c["B"], device=first.device)
    open_page = s["table"].long()[seq, first // page]              # the page it falls into, with first % page tokens
    kept = torch.arange(page, device=first.device)[None, :] < (first % page)[:, None]
    for n, x in (("k", _plain_rotate(s["k"].to(F32).view(T, nkv, d), pos, s)), ("v", s["v"].to(F32).view(T, nkv, d))):
        codes, scale = s[n + "_codes"], s[n + "_scale"]
        top = torch.zeros_like(scale).index_reduce_(0, blocks, x.abs().amax(dim=-1), "amax")
        fresh = torch.zeros(scale.shape[0], dtype=torch.bool, device=scale.device)
        fresh[blocks] = True
        fresh[open_page] = first % page == 0
        old = torch.where(fresh[:, None], torch.zeros_like(scale), scale)
        grown = torch.maximum(old, _scale_of(top))
        # the codes that an open page already holds follow its scale
        was = codes.view(torch.uint8)[open_page].view(F8)
        ratio = torch.where(grown[open_page] > 0, old[open_page] / grown[open_page], torch.ones_like(old[open_page]))
        now = (was.to(F32) * ratio[..., None, None]).to(F8)
        put = torch.where(kept[:, None, :, None], now.view(torch.uint8), was.view(torch.uint8))
        codes.view(torch.uint8)[open_page] = put
        touched = torch.zeros_like(fresh)
        touched[blocks] = True
        scale.copy_(torch.where(touched[:, None], grown, scale))
        by = scale[blocks][..., None]
        new = torch.where(by > 0, x / by, torch.zeros_like(x)).to(F8).view(torch.uint8)
        codes.view(torch.uint8)[blocks, :, pos % page] = new
    return {"k": s["k_codes"], "v": s["v_codes"], "k_scale": s["k_scale"], "v_scale": s["v_scale"], "q": s["q_out"]}


def _plain_attention(s):
    c = s["case"]
    B, nh, nkv, d, page, N = c["B"], c["nh"], c["nkv"], c["d"], c["page"], s["max_new"]
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
    last = s["seq_len"].long()[:, None] - new[:, None] + i[None, :]  # the last position a token sees
    seen = torch.arange(L, device=start.device)[None, None, :] <= last[:, :, None]
    score = score.view(B, nkv, nh // nkv, N, L).masked_fill(~seen[:, None, None], -math.inf)
    p = torch.exp(score - score.amax(dim=-1, keepdim=True).clamp(min=-3e38))
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.view(B, nkv, -1, L), cached("v")).view(B, nkv, nh // nkv, N, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    b, i, _ = _rows_of(s, T)
    s["o"].copy_(o.permute(0, 3, 1, 2, 4)[b, i].reshape(T, nh * d))
    return s["o"]


# ------------------------------------------------------------------ 64 bits

def _exact_rotate(x, pos, s, inverse=False):
    """Pair by pair as complex numbers."""
    c = s["case"]
    rot = c["rot"]
    turn = torch.polar(torch.full((pos.numel(), rot // 2), float(s["magnitude"]), dtype=F64, device=x.device),
                       torch.outer(pos.to(F64), s["freq"]) * (-1.0 if inverse else 1.0))
    x = x.to(F64).clone()
    one = slice(0, rot, 2) if c["interleaved"] else slice(0, rot // 2)
    two = slice(1, rot, 2) if c["interleaved"] else slice(rot // 2, rot)
    z = torch.complex(x[..., one].contiguous(), x[..., two].contiguous()) * turn[:, None, :]
    x[..., one], x[..., two] = z.real, z.imag
    return x


def _exact_e4m3(x):
    """The nearest e4m3 number, ties to the even one, for |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        return _exact_rotate(s["x"].view(c["T"], c["nh"], c["d"]) if c["gap"] == 0 else
                             s["x"].unflatten(1, (c["nh"], c["d"])), s["pos"], s, c["inverse"]).flatten(1)
    lens, news = _spans(c)
    nkv, d, page, nh = c["nkv"], c["d"], c["page"], c["nh"]
    T = sum(news)
    table = s["table"].cpu().tolist()
    if c["op"] == "append":
        pos = torch.cat([torch.arange(n - k, n) for n, k in zip(lens, news)]).to(s["q"].device)
        keys = _exact_rotate(s["k"].unflatten(1, (nkv, d)), pos, s)
        codes, scale = s["v_codes"].to(F64), {n: s[n + "_scale"].to(F64) for n in "kv"}
        at = 0
        for b, (n, k) in enumerate(zip(lens, news)):
            for page_no in range((n - k) // page, (n - 1) // page + 1):
                lo, hi = max(n - k, page_no * page), min(n, (page_no + 1) * page)
                p, old = table[b][page_no], lo % page
                rows = slice(at + lo - (n - k), at + hi - (n - k))
                for name, x in (("k", keys[rows]), ("v", s["v"][rows].unflatten(1, (nkv, d)).to(F64))):
                    part, power = torch.frexp(x.abs().amax(dim=(0, 2)) / E4M3_MAX)  # part 2^power, 1/2 <= part < 1
                    want = torch.exp2((power - (part == 0.5).to(power.dtype)).to(F64).clamp(min=MIN_EXP))
                    want = torch.where(part > 0, want, 0.0)
                    now = torch.maximum(want, scale[name][p]) if old else want
                    if name == "v":
                        by = torch.where(now > 0, now, 1.0)
                        codes[p, :, :old] = _exact_e4m3(codes[p, :, :old] * (scale[name][p] / by)[:, None, None])
                        codes[p, :, old:old + hi - lo] = _exact_e4m3(x / by[None, :, None]).transpose(0, 1)
                    scale[name][p] = now
            at += k
        # A rotated key within 32 bits' rounding of a border between two e4m3 numbers falls to either side:
        # one key element in a million, by chance, so 64 bits do not say which side is nearer.  The values
        # are not rotated: their codes have to be these.
        return {"k": None, "v": codes, "k_scale": scale["k"], "v_scale": scale["v"],
                "q": _exact_rotate(s["q"].view(T, nh, d), pos, s).flatten(1)}
    out, at = torch.zeros(T, nh, d, dtype=F64, device=s["q"].device), 0
    for b, (n, k) in enumerate(zip(lens, news)):
        pages = torch.tensor(table[b][:-(-n // page)], device=s["q"].device)
        for h in range(nkv):
            key, val = ((s[x + "_codes"].view(torch.uint8)[pages, h].view(F8).to(F64)
                         * s[x + "_scale"][pages, h].to(F64)[:, None, None]).reshape(-1, d)[:n] for x in "kv")
            heads = slice(h * (nh // nkv), (h + 1) * (nh // nkv))
            q = s["q"][at:at + k].to(F64).view(k, nh, d)[:, heads].transpose(0, 1)
            hidden = torch.ones(k, n, dtype=torch.bool, device=q.device).triu(n - k + 1)
            weight = torch.softmax((q @ key.T * d ** -0.5).masked_fill(hidden, -math.inf), dim=-1)
            out[at:at + k, heads] = (weight @ val).transpose(0, 1)
        at += k
    return out.flatten(1)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    c = case
    d = c["d"]
    if c["op"] == "rope":
        e = 2 if c["dtype"] == "bf16" else 4
        return {"bytes": 2 * c["T"] * c["nh"] * d * e + 4 * c["T"], "flops": 3 * c["T"] * c["nh"] * c["rot"]}
    lens, news = _spans(c)
    nh, nkv, page = c["nh"], c["nkv"], c["page"]
    T = sum(news)
    if c["op"] == "append":
        touched = sum((n - 1) // page - (n - k) // page + 1 for n, k in zip(lens, news))
        # keys and values in 16 bits, their codes, queries in and out, scales read and written
        bytes_ = T * nkv * d * 2 * 2 + T * nkv * d * 2 + 2 * T * nh * d * 2 + 2 * 2 * 4 * touched * nkv
        return {"bytes": bytes_, "flops": 3 * T * (nh + nkv) * c["rot"] + 2 * T * 2 * nkv * d}
    bytes_ = sum(2 * n * nkv * d + 2 * 4 * -(-n // page) * nkv for n in lens) + 2 * T * nh * d * 2
    flops = sum(4 * nh * d * (k * n - k * (k - 1) // 2) for n, k in zip(lens, news))
    return {"bytes": bytes_, "flops": flops}
