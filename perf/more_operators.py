"""Performance cases of what an attention block does around its quantized projections: what their users run, over the range of
sizes they run it at.

Three kinds of case (`op`):

cache      New keys and values of `B` sequences are written to a paged cache in 8 bits (a power-of-two scale for each 32 tokens of a
           head) and the blocks that they touched are read back.  A sequence brings `new` tokens and has `len` with them (`ragged`:
           up to that many, each sequence its own number).  `hk` heads of `D` entries, pages of `page` tokens; `fin`, `fout` are the
           types of what is written and read.
attn       Attention of the sequences' `new` last tokens over that cache: `hq` query heads for `hk` heads of keys and values.
           `causal`: a token sees itself and what is before it; `window` (0: none): only the last so many of them, and the
           sequence's first `sinks` tokens.
norm       The residual stream between two blocks: x + factor * gate * N(y), then a norm of it with its scale and shift for each
           sequence.  `M` rows of `C` features, `B` sequences; `after` and `norm` name the norms (none, rms, layer), `mod` whether
           gate, scale and shift are there, `fx`, `fy`, `fh` the types of the stream, of the block's output and of the normed rows.
"""
import math

import torch

own = False

BLOCK, E_MIN, E_MAX = 32, -20, 9      # tokens that share a scale 2^e, and the exponents a scale may have


def _cache(name, B, new, len, hk, D, page=64, ragged=False, fin="f16", fout="f16"):
    return {"name": name, "op": "cache", "B": B, "new": new, "len": len, "ragged": ragged, "hk": hk, "D": D, "page": page, "fin": fin,
            "fout": fout}


def _attn(name, B, new, len, hq, hk, D, causal=True, window=0, sinks=0, page=64, ragged=False):
    return {"name": name, "op": "attn", "B": B, "new": new, "len": len, "ragged": ragged, "hq": hq, "hk": hk, "D": D, "causal": causal,
            "window": window, "sinks": sinks, "page": page}


def _norm(name, M, C, B, after="none", norm="layer", mod=True, weight=False, fx="f16", fy="f16", fh="f16"):
    return {"name": name, "op": "norm", "M": M, "C": C, "B": B, "after": after, "norm": norm, "mod": mod, "weight": weight, "fx": fx, "fy": fy,
            "fh": fh}


def listed():
    return [
        # a step of 32 sequences, each with one new token far down the sequence: latency and scattered small writes
        _cache("cache-tokens-32", 32, 1, 4000, 8, 128, ragged=True),
        # five prompts of any length behind what their sequences hold already, fp32 rows, heads of the benchmark's blocks, small pages
        _cache("cache-ragged", 5, 1365, 2000, 16, 72, page=32, ragged=True, fin="f32", fout="f32"),
        # eight prompts of 4096 tokens at once
        _cache("cache-prompts", 8, 4096, 4096, 8, 128, page=128),
        # one new token of one short sequence: the smallest call
        _attn("attn-token", 1, 1, 300, 16, 16, 72),
        # a server's step: 64 sequences of many lengths, one new token each, four queries to a key
        _attn("attn-tokens-64", 64, 1, 8192, 32, 8, 128, ragged=True),
        # one sequence, far down: the long axis is all there is to share out
        _attn("attn-long", 1, 1, 131072, 32, 8, 128),
        # tokens that see a window and the first four, three tokens a step (two of them proposed), all heads of a group on one key
        _attn("attn-window-24", 24, 3, 20000, 10, 2, 80, window=1000, sinks=4, ragged=True),
        # prompts of any length with a window, in one call with short ones
        _attn("attn-ragged", 9, 1500, 5000, 28, 4, 112, window=2000, sinks=16, page=32, ragged=True),
        # the next part of a long prompt: 4096 tokens behind 4096
        _attn("attn-prompt", 1, 4096, 8192, 32, 8, 128),
        # the benchmark's images: two of 64 x 64 tokens, 16 heads of 72, every token sees every other
        _attn("attn-image", 2, 4096, 4096, 16, 16, 72, causal=False),
        # one row of one request
        _norm("norm-row", 1, 1152, 1),
        # eight images of 4096 tokens in the benchmark's wider blocks, fp32 stream, norm before and after the block
        _norm("norm-wide", 32768, 2240, 8, after="rms", norm="rms", weight=True, fx="f32"),
    ]


def _spread(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


_MOST_TOKENS = 8 * 4096 * 8 * 128           # entries of the keys that the largest listed cases write
_MOST_SEEN = 131072 * 8 * 128               # entries of the keys that they read
_MOST_PAIRS = 4096 * 6144 * 32 * 128        # products of queries and keys


def draw(rng):
    """1 .. 64 sequences of 1 .. 131072 tokens, 1 .. 8192 of them new; heads of 16 .. 256 entries; rows of 256 .. 8192 features."""
    kind = rng.choice(["cache", "attn", "attn", "norm"])
    if kind == "norm":
        C = 8 * round(_spread(rng, 256, 8192) / 8)
        M = max(1, min(round(_spread(rng, 1, 65536)), 32768 * 2240 // C))
        B = rng.choice([b for b in (1, 2, 3, 8, 16) if M % b == 0])
        c = _norm("", M, C, B, rng.choice(["none", "none", "rms", "layer"]), rng.choice(["rms", "layer"]), rng.random() < 0.7,
                  rng.random() < 0.5, *rng.choice([("f16", "f16", "f16"), ("f32", "f16", "f16"), ("f32", "f32", "f32"), ("f16", "f32", "f16")]))
        del c["name"]
        return c
    D = rng.choice([16, 40, 64, 64, 72, 80, 96, 112, 128, 128, 128, 192, 256])
    hk = rng.choice([1, 2, 4, 5, 8, 16])
    page = rng.choice([32, 64, 64, 128, 256])
    B = round(_spread(rng, 1, 64))
    if kind == "cache":
        new = max(1, min(round(_spread(rng, 1, 8192)), _MOST_TOKENS // (B * hk * D)))
        top = max(new, min(131072, _MOST_SEEN // (B * hk * D)))
        c = _cache("", B, new, round(_spread(rng, new, top)), hk, D, page, rng.random() < 0.7, *rng.choice([("f16", "f16"), ("f16", "f16"), ("f32", "f32")]))
    else:
        hq = hk * rng.choice([1, 1, 2, 4, 5, 7, 8])
        new = rng.choice([1, 1, 2, 5, round(_spread(rng, 2, 8192))])
        new = max(1, min(new, _MOST_TOKENS // (B * hk * D), _MOST_TOKENS // (B * hq * D), math.isqrt(_MOST_PAIRS // (B * hq * max(D, 64)))))
        top = max(new, min(131072, _MOST_SEEN // (B * hk * D), _MOST_PAIRS // (B * new * hq * max(D, 64))))
        causal = rng.random() < 0.8
        window = round(_spread(rng, 16, 8192)) if causal and rng.random() < 0.4 else 0
        c = _attn("", B, new, round(_spread(rng, new, top)), hq, hk, D, causal, window, rng.choice([0, 1, 4, 40]) if window else 0, page, rng.random() < 0.7)
    del c["name"]
    return c


_DTYPE = {"f16": torch.float16, "f32": torch.float32}


class _Held:
    """A library handle that is given back with the state that holds it."""

    def __init__(self, handle, free):
        self.h, self._free = handle, free

    def __del__(self):
        self._free(self.h)


# ---- sequences and their cache ---------------------------------------------------------------------------------------
def _lengths(case):
    """New tokens and tokens of each sequence: up to the case's, spread over the range."""
    B, new, top = case["B"], case["new"], case["len"]
    if not case["ragged"]:
        return [new] * B, [top] * B
    ns = [new - int((new - 1) * (0.7548776662 * i % 1.0)) for i in range(B)]
    return ns, [max(n, top - int((top - 1) * (0.6180339887 * i % 1.0))) for i, n in enumerate(ns)]


def _blocks(begins, ends, starts):
    """The blocks of 32 tokens that tokens begins[s] .. ends[s] - 1 of each sequence touch: sequence, block of the sequence, and the row of
    each of its 32 tokens in a list of them all (starts[s]: where the sequence's first one is), -1 where it is none of them."""
    seq, block, rows = [], [], []
    for s, (b, e, at) in enumerate(zip(begins, ends, starts)):
        first, last = b // BLOCK, -(-e // BLOCK)
        t = torch.arange(first * BLOCK, last * BLOCK, device="cuda")
        rows.append(torch.where((t >= b) & (t < e), t - b + at, -1).view(-1, BLOCK))
        seq.append(torch.full((last - first,), s, device="cuda"))
        block.append(torch.arange(first, last, device="cuda"))
    return torch.cat(seq), torch.cat(block), torch.cat(rows)


def _starts(ns):
    at = [0]
    for n in ns:
        at.append(at[-1] + n)
    return at


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _raw(case, g):
    """Keys and values of all tokens, sequence after sequence: heads of different sizes, a few entries of the keys far out; and the pages."""
    ns, lens = _lengths(case)
    T, H, D, P = sum(lens), case["hk"], case["D"], case["page"]
    dtype = _DTYPE[case.get("fin", "f16")]
    kv = []
    for far in (6.0, 1.0):
        x = torch.randn(T, H, D, generator=g, device="cuda", dtype=torch.float16).to(dtype)
        x *= 0.5 + torch.rand(1, H, 1, generator=g, device="cuda").to(dtype)
        x[..., torch.randperm(D, generator=g, device="cuda")[: max(1, D // 32)]] *= far
        kv.append(x)
    counts = [-(-n // P) for n in lens]
    order, at = torch.randperm(sum(counts), generator=g, device="cuda").to(torch.int32), 0
    pages = torch.zeros(len(lens), max(counts), dtype=torch.int32, device="cuda")
    for s, c in enumerate(counts):
        pages[s, :c] = order[at:at + c]
        at += c
    return kv, pages, sum(counts)


def _pow2(e):
    return ((e.int() + 127) << 23).view(torch.float32)


def _plain_write(s, rows, k, v):
    """Blocks of the cache with new tokens in them: the scale grows where they need a larger one, what was there is rounded to it."""
    at, new, before = rows
    for side, x in (("k", k), ("v", v)):
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, 1))[new].float()                     # [blocks][32][heads][D]; row -1: zeros
        frac, e = torch.frexp(x.abs().amax((1, 3)))
        need = (e - 7 + (frac > 127 / 128).int()).clamp(E_MIN, E_MAX)                       # smallest e with 127 * 2^e >= largest entry
        old, e_old = s[side + "codes"][at].float(), s[side + "exp"][at].int()
        e_old = torch.where(before.any(1)[:, None], e_old, E_MIN)
        e = torch.maximum(need, e_old)
        fresh = torch.round(x * _pow2(-e)[:, None, :, None]).clamp(-127, 127)
        kept = torch.round(old * _pow2(e_old - e)[:, None, :, None])
        codes = torch.where((new >= 0)[:, :, None, None], fresh, torch.where(before[:, :, None, None], kept, 0.0))
        s[side + "codes"][at] = codes.to(torch.int8)
        s[side + "exp"][at] = e.to(torch.int8)


def _plain_rows(s, seq, block, rows, begins):
    """What _plain_write goes by: places of the blocks in the cache, rows of their new tokens, which of their tokens were there before."""
    P = s["case"]["page"]
    per = P // BLOCK
    at = s["pages"][seq, block // per].long() * per + block % per
    t = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
    return at, rows, t < torch.tensor(begins, device="cuda")[seq][:, None]


def _fill(case, g, upto):
    """A state whose cache holds the first upto[s] tokens of each sequence, written at once."""
    (k, v), pages, n_pages = _raw(case, g)
    ns, lens = _lengths(case)
    H, D, P = case["hk"], case["D"], case["page"]
    s = {"op": case["op"], "case": case, "pages": pages, "uniform": len(set(ns)) == 1}
    s["length"], s["row_start"], s["rows"] = _ints(lens), _ints(_starts(ns)), sum(ns)
    there = torch.cat([torch.arange(a, a + u, device="cuda") for a, u in zip(_starts(lens), upto)])
    old_k, old_v, old_start = k[there], v[there], _ints(_starts(upto))
    if own:
        from paper_2604_18117_b200 import binding as L
        s["cache"] = _Held(L.lq_kvcache_create(1, n_pages, P, H, D, 0), L.lq_kvcache_free)
        s["dtype"] = {"f16": L.OUT_F16, "f32": L.OUT_F32}
        if len(there):
            length = _ints(upto)
            batch = L.lq_kvbatch(case["B"], len(there), length.data_ptr(), pages.data_ptr(), pages.shape[1], old_start.data_ptr())
            rows = L.lq_kvrows(old_k.data_ptr(), (0, H * D, D), old_v.data_ptr(), (0, H * D, D))
            L.lq_kvcache_append(s["cache"].h, 0, batch, rows, s["dtype"][case.get("fin", "f16")], torch.cuda.current_stream().cuda_stream)
    else:
        for side in "kv":
            s[side + "codes"] = torch.zeros(n_pages * P // BLOCK, BLOCK, H, D, dtype=torch.int8, device="cuda")
            s[side + "exp"] = torch.zeros(n_pages * P // BLOCK, H, dtype=torch.int8, device="cuda")
        if len(there):
            seq, block, rows = _blocks([0] * len(upto), upto, _starts(upto))
            for part in torch.arange(len(seq), device="cuda").split(1 << 12):
                _plain_write(s, _plain_rows(s, seq[part], block[part], rows[part], [0] * len(upto)), old_k, old_v)
    return s, k, v


def _batch(L, s):
    """The sequences of a step; where all bring the same number of tokens, that is all there is to say."""
    return L.lq_kvbatch(s["case"]["B"], s["rows"], s["length"].data_ptr(), s["pages"].data_ptr(), s["pages"].shape[1],
                        None if s["uniform"] else s["row_start"].data_ptr())


# ---- cache -----------------------------------------------------------------------------------------------------------
def _prepare_cache(case, g):
    ns, lens = _lengths(case)
    begins = [t - n for t, n in zip(lens, ns)]
    s, k, v = _fill(case, g, begins)
    new = torch.cat([torch.arange(a + b, a + t, device="cuda") for a, b, t in zip(_starts(lens), begins, lens)])
    s["k"], s["v"] = k[new], v[new]
    firsts = [b // BLOCK * BLOCK for b in begins]
    most = max(t - f for t, f in zip(lens, firsts))
    s["most"] = most
    if own:
        s["begin"] = _ints(firsts)
        for side in "kv":
            s[side + "_out"] = torch.zeros(case["B"], most, case["hk"], case["D"], dtype=_DTYPE[case["fout"]], device="cuda")
    else:
        seq, block, rows = _blocks(begins, lens, _starts(ns))
        s["write"] = _plain_rows(s, seq, block, rows, begins)
        t = block[:, None] * BLOCK + torch.arange(BLOCK, device="cuda")
        slot = seq[:, None] * most + t - torch.tensor(firsts, device="cuda")[seq][:, None]
        s["slot"] = torch.where(t < s["length"][seq][:, None], slot, case["B"] * most).flatten()
    return s


def _plain_cache(s):
    case = s["case"]
    _plain_write(s, s["write"], s["k"], s["v"])
    outs = {}
    for side in "kv":
        at = s["write"][0]
        x = s[side + "codes"][at].float() * _pow2(s[side + "exp"][at])[:, None, :, None]
        y = torch.zeros(case["B"] * s["most"] + 1, case["hk"], case["D"], device="cuda")
        y[s["slot"]] = x.flatten(0, 1)
        outs[side] = y[:-1].view(case["B"], s["most"], case["hk"], case["D"]).to(_DTYPE[case["fout"]])
    return outs


def _own_cache(L, s, stream):
    case = s["case"]
    H, D = case["hk"], case["D"]
    batch = _batch(L, s)
    L.lq_kvcache_append(s["cache"].h, 0, batch, L.lq_kvrows(s["k"].data_ptr(), (0, H * D, D), s["v"].data_ptr(), (0, H * D, D)),
                        s["dtype"][case["fin"]], stream)
    strides = (s["most"] * H * D, H * D, D)
    L.lq_kvcache_read(s["cache"].h, 0, batch, s["begin"].data_ptr(), s["most"], L.lq_kvrows(s["k_out"].data_ptr(), strides, s["v_out"].data_ptr(), strides),
                      s["dtype"][case["fout"]], stream)
    return {"k": s["k_out"], "v": s["v_out"]}


def _exact_step(x):
    """Step 2^e of each block and head of x [blocks][32][heads][D]."""
    steps = torch.tensor([2.0 ** e for e in range(E_MIN, E_MAX + 1)], dtype=torch.float64, device="cuda")
    i = torch.searchsorted(127 * steps, x.abs().amax((1, 3)).contiguous()).clamp(max=len(steps) - 1)       # the smallest that does not clip
    return steps[i][:, None, :, None]


def _exact_held(x, before):
    """What a cache holds of one sequence's keys or values x [tokens][heads][D], of which the first `before` were written first."""
    T, H, D = x.shape
    t = torch.arange(-(-T // BLOCK) * BLOCK, device="cuda").view(-1, BLOCK, 1, 1)
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, t.numel() - T)).double().view(-1, BLOCK, H, D)
    step = _exact_step(torch.where(t < before, x, 0.0))
    held = (x / step).round().clamp(-127, 127) * step
    step = torch.maximum(step, _exact_step(torch.where(t < before, 0.0, x)))
    held = torch.where(t < before, held / step, (x / step).clamp(-127, 127)).round() * step
    return held.flatten(0, 1)[:T]


def _exact_cache(case, seed):
    (k, v), _, _ = _raw(case, torch.Generator(device="cuda").manual_seed(seed))
    ns, lens = _lengths(case)
    firsts = [(t - n) // BLOCK * BLOCK for n, t in zip(ns, lens)]
    outs = {}
    for side, x in (("k", k), ("v", v)):
        outs[side] = torch.zeros(case["B"], max(t - f for t, f in zip(lens, firsts)), case["hk"], case["D"], dtype=torch.float64, device="cuda")
        for i, (a, n, t, f) in enumerate(zip(_starts(lens), ns, lens, firsts)):
            outs[side][i, : t - f] = _exact_held(x[a + f:a + t], t - n - f)
    return outs


# ---- attn ------------------------------------------------------------------------------------------------------------
def _prepare_attn(case, g):
    ns, lens = _lengths(case)
    s, _, _ = _fill(case, g, lens)
    # queries as they lie in a projection's rows, in front of keys and values
    qkv = torch.randn(sum(ns), case["hq"] + 2 * case["hk"], case["D"], generator=g, device="cuda", dtype=torch.float16)
    s["q"] = qkv[:, : case["hq"]]
    s["out"] = torch.empty(sum(ns), case["hq"], case["D"], dtype=torch.float16, device="cuda")
    if not own:
        # a sequence's rows, filled up to the longest; where each row is in that
        s["pad"] = torch.nn.utils.rnn.pad_sequence([torch.arange(a, a + n) for a, n in zip(_starts(ns), ns)], batch_first=True, padding_value=sum(ns)).cuda()
        s["place"] = torch.cat([torch.arange(n) + i * max(ns) for i, n in enumerate(ns)]).cuda()
        s["pos"] = (torch.tensor(lens) - torch.tensor(ns))[:, None].cuda() + torch.arange(max(ns), device="cuda")
        s["top"] = max(lens)
    return s


def _plain_attn(s):
    case = s["case"]
    hk, D, P = case["hk"], case["D"], case["page"]
    g = case["hq"] // hk
    t = torch.arange(s["top"], device="cuda")
    at = s["pages"][:, t // P].long() * (P // BLOCK) + t % P // BLOCK                       # [B][tokens]

    def held(side):                                      # [B][hk][tokens][D]
        return (s[side + "codes"][at, t % BLOCK].float() * _pow2(s[side + "exp"][at])[..., None]).transpose(1, 2)

    q = torch.nn.functional.pad(s["q"], (0, 0, 0, 0, 0, 1))[s["pad"]].float()               # [B][rows][hq][D]
    B, n = q.shape[:2]
    q = q.view(B, n, hk, g, D).permute(0, 2, 3, 1, 4).reshape(B, hk, g * n, D) / math.sqrt(D)
    p = torch.matmul(q, held("k").transpose(2, 3)).view(B, hk, g, n, -1)
    pos, seen = s["pos"][:, :, None], t[None, None] < s["length"][:, None, None]
    if case["causal"]:
        seen = seen & (t <= pos)
    if case["window"]:
        seen = seen & ((t > pos - case["window"]) | (t < case["sinks"]))
    p = p.masked_fill_(~seen[:, None, None], -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    y = torch.matmul(p.view(B, hk, g * n, -1), held("v")).view(B, hk, g, n, D) / total
    return y.permute(0, 3, 1, 2, 4).reshape(B * n, case["hq"], D)[s["place"]].half()


def _own_attn(L, s, stream):
    case = s["case"]
    a = L.lq_attn(s["q"].data_ptr(), s["q"].stride()[:2], s["out"].data_ptr(), s["out"].stride()[:2], case["hq"], 1 / math.sqrt(case["D"]),
                  case["causal"], case["window"], case["sinks"])
    L.lq_cache_attention(s["cache"].h, 0, _batch(L, s), a, stream)
    return s["out"]


def _exact_attn(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    (k, v), _, _ = _raw(case, g)
    ns, lens = _lengths(case)
    q = torch.randn(sum(ns), case["hq"] + 2 * case["hk"], case["D"], generator=g, device="cuda", dtype=torch.float16)[:, : case["hq"]]
    out = torch.empty(sum(ns), case["hq"], case["D"], dtype=torch.float64, device="cuda")
    group = case["hq"] // case["hk"]
    for a, b, n, t in zip(_starts(lens), _starts(ns), ns, lens):
        ks, vs = _exact_held(k[a:a + t], t), _exact_held(v[a:a + t], t)
        j = torch.arange(t, device="cuda")
        for h in range(case["hq"]):
            for part in torch.arange(n, device="cuda").split(1024):
                i = part[:, None] + (t - n)
                x = q[b + part, h].double() @ ks[:, h // group].T * case["D"] ** -0.5
                if case["causal"]:
                    near = (j > i - case["window"]) | (j < case["sinks"]) if case["window"] else j >= 0
                    x = torch.where((j <= i) & near, x, -math.inf)
                out[b + part, h] = torch.softmax(x, -1) @ vs[:, h // group]
    return out


# ---- norm ------------------------------------------------------------------------------------------------------------
def _prepare_norm(case, g):
    M, C, B = case["M"], case["C"], case["B"]
    x = torch.randn(M, C, generator=g, device="cuda") * 2
    x[:, torch.randperm(C, generator=g, device="cuda")[: max(1, C // 100)]] *= 15           # a stream's few large features
    s = {"op": "norm", "case": case, "x": x.to(_DTYPE[case["fx"]])}
    del x
    s["y"] = torch.randn(M, C, generator=g, device="cuda").to(_DTYPE[case["fy"]])
    s["x_out"], s["h"] = torch.empty_like(s["x"]), torch.empty(M, C, dtype=_DTYPE[case["fh"]], device="cuda")
    # six vectors of each sequence as a conditioning projection puts them out; these operators use three of them
    s["mod"] = (0.3 * torch.randn(B, 6, C, generator=g, device="cuda")).half() if case["mod"] else None
    for name in ("w_after", "w"):
        s[name] = 1 + 0.2 * torch.randn(C, generator=g, device="cuda") if case["weight"] else None
    s["factor"] = 1.0 if case["mod"] else 0.5
    return s


_EPS = 1e-6


def _plain_normed(x, kind, w):
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    if kind != "none":
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS)
        x = x if w is None else x * w
    return x


def _plain_norm(s):
    case = s["case"]
    M, C, B = case["M"], case["C"], case["B"]
    y = _plain_normed(s["y"].float(), case["after"], s["w_after"]).view(B, M // B, C)
    mod = None if s["mod"] is None else s["mod"].float()[:, :, None]
    y = s["factor"] * (y if mod is None else y * mod[:, 2])
    x = s["x"].float().view(B, M // B, C) + y
    h = _plain_normed(x, case["norm"], s["w"])
    h = h if mod is None else h * (1 + mod[:, 1]) + mod[:, 0]
    return {"x": x.view(M, C).to(_DTYPE[case["fx"]]), "h": h.view(M, C).to(_DTYPE[case["fh"]])}


def _own_norm(L, s, stream):
    case = s["case"]
    code = {"f16": L.OUT_F16, "f32": L.OUT_F32}
    kind = {"none": L.NORM_NONE, "rms": L.NORM_RMS, "layer": L.NORM_LAYER}
    ptr = lambda t: None if t is None else t.data_ptr()                                      # noqa: E731
    mod = [None] * 3 if s["mod"] is None else [s["mod"][:, i].data_ptr() for i in range(3)]
    r = L.lq_residual(case["M"], case["C"], s["x"].data_ptr(), s["x_out"].data_ptr(), s["h"].data_ptr(), y_ptr=s["y"].data_ptr(),
                      sequences=case["B"], after=kind[case["after"]], after_weight_ptr=None if case["after"] == "none" else ptr(s["w_after"]), factor=s["factor"],
                      gate_ptr=mod[2], norm=kind[case["norm"]], weight_ptr=ptr(s["w"]), shift_ptr=mod[0], scale_ptr=mod[1],
                      mod_seq=6 * case["C"], eps=_EPS, x_dtype=code[case["fx"]], y_dtype=code[case["fy"]], h_dtype=code[case["fh"]],
                      mod_dtype=L.OUT_F16)
    L.lq_residual_norm(r, stream)
    return {"x": s["x_out"], "h": s["h"]}


def _exact_norm(case, seed):
    s = _prepare_norm(case, torch.Generator(device="cuda").manual_seed(seed))
    M, B = case["M"], case["B"]

    def normed(x, kind, w):
        if kind == "none":
            return x
        x = x - x.mean(-1, keepdim=True) if kind == "layer" else x
        x = x * ((x * x).sum(-1, keepdim=True) / x.shape[-1] + _EPS).rsqrt()
        return x if w is None else x * w.double()

    outs = {"x": torch.empty(M, case["C"], dtype=torch.float64, device="cuda"), "h": torch.empty(M, case["C"], dtype=torch.float64, device="cuda")}
    for rows in torch.arange(M, device="cuda").split(4096):
        mod = None if s["mod"] is None else s["mod"].double()[rows * B // M]
        y = normed(s["y"][rows].double(), case["after"], s["w_after"]) * s["factor"]
        x = s["x"][rows].double() + (y if mod is None else mod[:, 2] * y)
        h = normed(x, case["norm"], s["w"])
        outs["x"][rows], outs["h"][rows] = x, h if mod is None else h + mod[:, 1] * h + mod[:, 0]
    return outs


# ---- what is called ----------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return {"cache": _prepare_cache, "attn": _prepare_attn, "norm": _prepare_norm}[case["op"]](case, g)


def run(state):
    if own:
        from paper_2604_18117_b200 import binding as L
        stream = torch.cuda.current_stream().cuda_stream
        return {"cache": _own_cache, "attn": _own_attn, "norm": _own_norm}[state["op"]](L, state, stream)
    return {"cache": _plain_cache, "attn": _plain_attn, "norm": _plain_norm}[state["op"]](state)


def exact(case, seed):
    return {"cache": _exact_cache, "attn": _exact_attn, "norm": _exact_norm}[case["op"]](case, seed)


def _seen(case, i, t):
    """Tokens that the new token at place i of t sees."""
    if not case["causal"]:
        return t
    if not case["window"] or i < case["window"]:
        return i + 1
    return case["window"] + min(case["sinks"], i + 1 - case["window"])


def work(case):
    """Cache: new rows in, codes out, the blocks that they touch read back; what was in those before in and out.  Attention: the tokens
    that any new token sees, once, with their scales, queries in, outputs out; two products for each pair.  Norm: the stream in and out,
    the block's output in, normed rows out, and the vectors; some ten operations an entry."""
    size = {"f16": 2, "f32": 4}
    if case["op"] == "norm":
        n = case["M"] * case["C"]
        extra = 6 * case["B"] * case["C"] if case["mod"] else 0
        return {"bytes": n * (2 * size[case["fx"]] + size[case["fy"]] + size[case["fh"]]) + extra + (8 * case["C"] if case["weight"] else 0), "flops": 10 * n}
    ns, lens = _lengths(case)
    H, D = case["hk"], case["D"]
    scales = 2 * H / BLOCK
    if case["op"] == "cache":
        touched = sum(t - (t - n) // BLOCK * BLOCK for n, t in zip(ns, lens))
        new = sum(ns)
        nbytes = 2 * H * D * (new * (size[case["fin"]] + 1) + touched * (1 + size[case["fout"]])) + touched * scales
        return {"bytes": int(nbytes), "flops": 4 * 2 * H * D * (new + touched)}
    pairs, tokens = 0, 0
    for n, t in zip(ns, lens):
        pairs += sum(_seen(case, i, t) for i in range(t - n, t)) if case["causal"] else n * t
        first = max(0, t - n - case["window"] + 1) if case["window"] else 0                 # of the window of the first new token
        tokens += t - first + min(case["sinks"], first)
    return {"bytes": int(tokens * (2 * H * D + scales) + 4 * sum(ns) * case["hq"] * D), "flops": 4 * pairs * case["hq"] * D}
