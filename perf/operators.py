"""Performance cases of the operators around the quantized projections: what their users run, over the range of sizes they
run it at.

Two kinds of case (`op`):

adapters   Y = Y0 + scale_a (X A_a) B_a, row by row with the low-rank adapter a that the row's request has chosen (or none),
           beside a shared projection whose output is Y0.  `shapes` lists the projections as "KxN" (one map of rows serves all of
           them, as a step of a program has it), `M` the rows, `slots` the adapters that are loaded, `rank` the largest rank
           (`mixed`: the adapters' ranks differ), `runs` the requests of neighbouring rows (0: each row is a request of its own,
           in any order), `none_every`: every such run or row has no adapter (0: all have one), `out` the type of Y0 and Y.
heads      Queries and keys of `B` sequences of `S` rows: a norm of each head (`norm`: rms, layer or none), then the rotation of
           its leading entries by the row's position on one to four axes.  `dims` lists the entries of each axis, `order` says
           whether each axis has frequencies of its own ("split") or the axes share out one head's ("shared"), `layout`
           whether a pair is two neighbours ("pairs") or entries half of the rotated part apart ("halves").  `grid` is the
           extent of the axes (positions count through it, last axis fastest), `far` the largest offset of an axis, `src` whether
           Q and K lie in a fused projection's rows ("qkv") or by themselves ("own"), `dst` the order of the outputs.
"""
import math

import torch

own = False


def _adapters(name, shapes, M, slots, rank, runs, mixed=False, none_every=0, out="f16"):
    return {"name": name, "op": "adapters", "shapes": shapes, "M": M, "slots": slots, "rank": rank, "mixed": mixed, "runs": runs,
            "none_every": none_every, "out": out}


def _heads(name, B, S, hq, hk, D, norm, dims, grid, order="split", layout="pairs", theta=10000.0, far=0, src="qkv", dst="bshd",
           weight=True, fin="f16", fout="f16"):
    return {"name": name, "op": "heads", "B": B, "S": S, "hq": hq, "hk": hk, "D": D, "norm": norm, "weight": weight, "dims": dims,
            "grid": grid, "order": order, "layout": layout, "theta": theta, "far": far, "src": src, "dst": dst, "fin": fin, "fout": fout}


PIXART = "1152x3456,1152x1152,1152x4608,4608x1152"      # the four linears of the benchmark's block (hidden 1152, MLP 4608)


def listed():
    return [
        # one conditioning vector of one request through a projection: launches and latency are all there is
        _adapters("adapters-row", "1152x1152", 1, 4, 16, 1),
        # a batch of single rows, each with an adapter of its own (a pooled vector of each request, a step of a decoder):
        # every adapter is read for one row
        _adapters("adapters-rows-64", "1152x4608", 64, 64, 32, 0),
        # no size a multiple of a tile, ranks that differ, rows of a few requests in any order, some without an adapter, fp32
        _adapters("adapters-ragged-1365", "1160x2312", 1365, 7, 24, 0, mixed=True, none_every=5, out="f32"),
        # eight image requests of 1024 tokens through a block's four linears, three adapters loaded
        _adapters("adapters-block", PIXART, 8192, 3, 32, 8),
        # the benchmark's largest batch through the widest factors: 8 requests of 4096 tokens, an MLP's second linear
        _adapters("adapters-wide", "5600x2240", 32768, 8, 128, 8),
        # one token of one request: the smallest call
        _heads("heads-row", 1, 1, 16, 16, 72, "rms", "72", "1", far=4000, layout="halves"),
        # Q and K of the benchmark's qkv linear, two images of 64 x 64 tokens, 16 heads of 72, rows and columns as two axes
        _heads("heads-image", 2, 4096, 16, 16, 72, "rms", "36,36", "64,64"),
        # ragged: fp32 rows, LayerNorm, heads of 112 rotated in part, four queries to a key, far positions
        _heads("heads-ragged", 3, 455, 20, 5, 112, "layer", "96", "455", layout="halves", far=900000, fin="f32"),
        # 32 sequences with one new token each, far down the sequence
        _heads("heads-tokens-32", 32, 1, 32, 8, 128, "rms", "128", "1", layout="halves", theta=1e6, far=120000),
        # video: 21 x 30 x 52 tokens, each axis with frequencies of its own, heads apart in memory as an attention kernel has them
        _heads("axes-video", 1, 32760, 20, 20, 128, "rms", "44,42,42", "21,30,52", dst="bhsd"),
        # images and text in one sequence: three axes share out one head's frequencies, no norm, fp32 in and out
        _heads("axes-shared", 2, 2050, 28, 4, 128, "none", "32,48,48", "2,25,41", order="shared", layout="halves", theta=1e6,
               far=9000, fin="f32", fout="f32", src="own"),
    ]


def _spread(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


_MOST_ADAPTERS = 32768 * (5600 + 2 * 2240)             # halves of X, Y0 and Y in the largest listed case


def draw(rng):
    """M over 1 .. 32768 rows, K and N over 256 .. 8192 in steps of 8, ranks 1 .. 128, up to 64 adapters; heads of 32 .. 256 entries."""
    if rng.random() < 0.5:
        K, N = (8 * round(_spread(rng, 256, 8192) / 8) for _ in range(2))
        out = rng.choice(["f16", "f16", "f32"])
        M = max(1, min(round(_spread(rng, 1, 32768)), _MOST_ADAPTERS // (K + 2 * N * (2 if out == "f32" else 1))))
        slots = round(_spread(rng, 1, 64))
        c = _adapters("", f"{K}x{N}", M, slots, rng.choice([1, 8, 13, 16, 24, 32, 32, 48, 64, 100, 128]),
                      rng.choice([0, min(M, round(_spread(rng, 1, 64)))]), rng.random() < 0.5, rng.choice([0, 0, 3, 7]), out)
    else:
        D = rng.choice([32, 40, 64, 72, 80, 96, 112, 128, 128, 160, 256])
        axes = rng.choice([1, 1, 2, 3, 4])
        cut = sorted(2 * rng.randint(1, D // 2 - 1) for _ in range(axes - 1)) + [D if axes > 1 else rng.choice([D, 16, 24])]
        dims = [b - a for a, b in zip([0] + cut, cut)]
        hk = rng.choice([1, 2, 5, 8, 16])
        hq = hk * rng.choice([1, 1, 2, 4])
        fin = rng.choice(["f16", "f16", "f32"])
        most = 32760 * 40 * 128 // ((hq + hk) * D * (1 if fin == "f16" else 2))            # rows of the largest listed case
        S = max(1, min(round(_spread(rng, 1, 32768)), most))
        B = max(1, min(rng.choice([1, 1, 2, 3, 16]), 32768 // S, most // S))
        c = _heads("", B, S, hq, hk, D, rng.choice(["rms", "rms", "layer", "none"]), ",".join(str(max(0, d)) for d in dims),
                   ",".join(str(rng.choice([3, 17, 64])) for _ in range(axes)), rng.choice(["split", "shared"]),
                   rng.choice(["pairs", "halves"]), rng.choice([100.0, 10000.0, 1e6]), rng.choice([0, 100, 1000000]),
                   rng.choice(["qkv", "own"]), rng.choice(["bshd", "bhsd"]), rng.random() < 0.7, fin,
                   "f16" if fin == "f16" else rng.choice(["f16", "f32"]))
    del c["name"]
    return c


_DTYPE = {"f16": torch.float16, "f32": torch.float32}


class _Held:
    """A library handle that is given back with the state that holds it."""

    def __init__(self, handle, free):
        self.h, self._free = handle, free

    def __del__(self):
        self._free(self.h)


# ---- adapters --------------------------------------------------------------------------------------------------------
def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def _ranks(case):
    """Ranks of the adapters in the slots."""
    r = case["rank"]
    return [max(1, (r, r // 2, 3 * r // 4, 1, r)[s % 5]) if case["mixed"] else r for s in range(case["slots"])]


def _requests(case):
    """Adapter of each request (a run of rows, or a row); -1: none."""
    n, every = case["runs"] or case["M"], case["none_every"]
    return [-1 if every and i % every == every - 1 else i % case["slots"] for i in range(n)]


def _prepare_adapters(case, g):
    M, slots = case["M"], case["slots"]
    req = torch.tensor(_requests(case), dtype=torch.int32)
    if case["runs"]:                                     # requests of about the same length, one behind the other
        row = torch.div(torch.arange(M) * case["runs"], M, rounding_mode="floor")
        ids = req[row].cuda()
    else:
        ids = req.cuda()[torch.randperm(M, generator=g, device="cuda")]
    # the rows of each adapter that is in use, as a program's scheduler has them; short lists are filled up with row M
    host = ids.cpu()
    used = [s for s in range(slots) if bool((host == s).any())]
    lists = [torch.nonzero(host == s)[:, 0] for s in used] or [torch.zeros(0, dtype=torch.int64)]
    groups = torch.nn.utils.rnn.pad_sequence(lists, batch_first=True, padding_value=M).cuda()
    ranks = _ranks(case)
    state = {"op": "adapters", "M": M, "ids": ids, "groups": groups, "used": torch.tensor(used or [0], device="cuda"), "linears": []}
    state["scale"] = torch.tensor([1.0 + 0.125 * (s % 4) for s in range(slots)], device="cuda")
    live = torch.arange(case["rank"], device="cuda")[None] < torch.tensor(ranks, device="cuda")[:, None]      # [slots][rank]
    for K, N in _shapes(case):
        x = torch.randn(M, K, generator=g, device="cuda")
        if K > 4000:                                     # behind an activation function values lean to one side
            x = torch.nn.functional.gelu(x)
        x[:, torch.randperm(K, generator=g, device="cuda")[: max(8, K // 100)]] *= 20
        lin = {"X": x.half(), "Y0": torch.randn(M, N, generator=g, device="cuda").to(_DTYPE[case["out"]])}
        del x
        a = torch.randn(slots, K, case["rank"], generator=g, device="cuda") * (0.2 / math.sqrt(K))
        b = torch.randn(slots, case["rank"], N, generator=g, device="cuda") * 0.3
        lin["A"], lin["B"] = (a * live[:, None]).half(), (b * live[:, :, None]).half()
        lin["Y"] = torch.empty_like(lin["Y0"])
        state["linears"].append(lin)
    if own:
        from paper_2604_18117_b200 import binding as L
        stream = torch.cuda.current_stream().cuda_stream
        state["map"] = _Held(L.lq_rowmap_create(M, slots, 0), L.lq_rowmap_free)
        state["out"] = L.OUT_F32 if case["out"] == "f32" else L.OUT_F16
        for (K, N), lin in zip(_shapes(case), state["linears"]):
            lin["set"] = _Held(L.lq_adapters_create(K, N, case["rank"], slots, 0), L.lq_adapters_free)
            for s, r in enumerate(ranks):
                A, B = lin["A"][s, :, :r].contiguous(), lin["B"][s, :r].contiguous()
                L.lq_adapters_set(lin["set"].h, s, r, A.data_ptr(), B.data_ptr(), float(state["scale"][s]), stream)
    return state


def _plain_adapters(s, lin):
    groups, used = s["groups"], s["used"]
    X = torch.nn.functional.pad(lin["X"], (0, 0, 0, 1))[groups].float()
    D = torch.bmm(torch.bmm(X, lin["A"][used].float()), lin["B"][used].float()) * s["scale"][used][:, None, None]
    Y = torch.nn.functional.pad(lin["Y0"], (0, 0, 0, 1)).float()
    Y[groups] = Y[groups] + D
    return Y[:-1].to(lin["Y0"].dtype)


def _own_adapters(L, s, lin, stream):
    L.lq_adapters_forward(lin["set"].h, s["map"].h, lin["X"].data_ptr(), lin["Y0"].data_ptr(), lin["Y"].data_ptr(), s["out"], stream)
    return lin["Y"]


def _exact_adapters(case, seed):
    s = _prepare_adapters(case, torch.Generator(device="cuda").manual_seed(seed))
    outs = []
    for (K, N), lin in zip(_shapes(case), s["linears"]):
        Y = lin["Y0"].double()
        for a in range(case["slots"]):
            rows = torch.nonzero(s["ids"] == a)[:, 0]
            for part in rows.split(4096):
                Y[part] += float(s["scale"][a]) * (lin["X"][part].double() @ lin["A"][a].double() @ lin["B"][a].double())
        outs.append(Y)
    return outs


# ---- heads -----------------------------------------------------------------------------------------------------------
def _ints(text):
    return [int(v) for v in text.split(",")]


def _pairs(case):
    """Axis and frequency (radians a position) of each rotated pair."""
    dims, theta = _ints(case["dims"]), case["theta"]
    axis = [a for a, d in enumerate(dims) for _ in range(d // 2)]
    if case["order"] == "shared":
        freq = [theta ** (-2.0 * i / sum(dims)) for i in range(sum(dims) // 2)]
    else:
        freq = [theta ** (-2.0 * i / d) for d in dims for i in range(d // 2)]
    return axis, freq


def _sides(case, state):
    """[("q", heads, input), ("k", ...)], inputs as [B][S][heads][D]."""
    hq, hk = case["hq"], case["hk"]
    if case["src"] == "own":
        return [("q", hq, state["q"]), ("k", hk, state["k"])]
    return [("q", hq, state["qkv"][:, :, :hq]), ("k", hk, state["qkv"][:, :, hq:hq + hk])]


def _prepare_heads(case, g):
    B, S, hq, hk, D = (case[k] for k in ("B", "S", "hq", "hk", "D"))

    def values(h):
        # what a projection puts out: heads of different sizes, a few entries far out
        x = torch.randn(B, S, h, D, generator=g, device="cuda") * (0.5 + torch.rand(1, 1, h, 1, generator=g, device="cuda"))
        x[..., torch.randperm(D, generator=g, device="cuda")[: max(1, D // 32)]] *= 8
        return x.to(_DTYPE[case["fin"]])

    state = {"op": "heads", "case": case}
    if case["src"] == "own":
        state["q"], state["k"] = values(hq), values(hk)
    else:
        state["qkv"] = values(hq + 2 * hk)               # V lies behind K and is left alone
    grid = _ints(case["grid"])
    at, pos = torch.arange(S, device="cuda"), []
    for n in reversed(grid):
        pos.append(at % n)
        at = torch.div(at, n, rounding_mode="floor")
    pos[-1] = pos[-1] + at * grid[0]                     # the slowest axis goes on where the grid is shorter than the sequence
    pos = torch.stack(pos[::-1], -1)[None].expand(B, S, len(grid))
    off = torch.randint(0, case["far"] + 1, (B, 1, len(grid)), generator=g, device="cuda")
    state["pos"] = (pos + off).to(torch.int32).contiguous()
    axis, freq = _pairs(case)
    state["axis"], state["freq"] = torch.tensor(axis, device="cuda"), torch.tensor(freq, dtype=torch.float64, device="cuda")
    for side in "qk":
        w = 1 + 0.2 * torch.randn(D, generator=g, device="cuda")
        b = 0.1 * torch.randn(D, generator=g, device="cuda")
        state["w" + side] = w if case["weight"] and case["norm"] != "none" else None
        state["b" + side] = b if case["weight"] and case["norm"] == "layer" else None
    for side, h, x in _sides(case, state):
        shape = (B, S, h, D) if case["dst"] == "bshd" else (B, h, S, D)
        state[side + "_out"] = torch.empty(shape, dtype=_DTYPE[case["fout"]], device="cuda")
    if own:
        from paper_2604_18117_b200 import binding as L
        cfg = L.lq_rope_config_default(_ints(case["dims"]), theta=case["theta"], halves=case["layout"] == "halves",
                                       shared=case["order"] == "shared")
        state["rope"] = _Held(L.lq_rope_create(cfg, 0), L.lq_rope_free)
        state["norm"] = {"none": L.NORM_NONE, "rms": L.NORM_RMS, "layer": L.NORM_LAYER}[case["norm"]]
    return state


def _plain_side(s, x, w, b, cos, sin):
    case = s["case"]
    x = x.float()
    if case["norm"] == "rms":
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    elif case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    x = x if w is None else x * w
    x = x if b is None else x + b
    P = cos.shape[-1]
    lo, hi = (x[..., :P], x[..., P:2 * P]) if case["layout"] == "halves" else (x[..., 0:2 * P:2], x[..., 1:2 * P:2])
    lo, hi = lo * cos - hi * sin, hi * cos + lo * sin
    turned = torch.cat([lo, hi], -1) if case["layout"] == "halves" else torch.stack([lo, hi], -1).flatten(-2)
    y = torch.cat([turned, x[..., 2 * P:]], -1)
    y = y if case["dst"] == "bshd" else y.transpose(1, 2)
    return y.to(_DTYPE[case["fout"]]).contiguous()


def _plain_heads(s):
    angle = s["pos"].double()[..., s["axis"]] * s["freq"]                  # far positions: angles need 64 bits
    cos, sin = (f(angle).float()[:, :, None] for f in (torch.cos, torch.sin))
    return {side: _plain_side(s, x, s["w" + side], s["b" + side], cos, sin) for side, h, x in _sides(s["case"], s)}


def _own_heads(L, s, stream):
    case = s["case"]
    code = {"f16": L.OUT_F16, "f32": L.OUT_F32}
    # strides over sequences, rows and heads, of the inputs as they lie and of the outputs in either order
    heads = {side: L.lq_heads(x.data_ptr(), x.stride()[:3], s[side + "_out"].data_ptr(),
                              [s[side + "_out"].stride(i) for i in ((0, 1, 2) if case["dst"] == "bshd" else (0, 2, 1))], h,
                              None if s["w" + side] is None else s["w" + side].data_ptr(),
                              None if s["b" + side] is None else s["b" + side].data_ptr()) for side, h, x in _sides(case, s)}
    L.lq_qk_norm_rope(heads["q"], heads["k"], case["D"], case["B"], case["S"], s["norm"], 1e-6, s["rope"].h, s["pos"].data_ptr(),
                      code[case["fin"]], code[case["fout"]], stream)
    return {"q": s["q_out"], "k": s["k_out"]}


def _exact_heads(case, seed):
    s = _prepare_heads(case, torch.Generator(device="cuda").manual_seed(seed))
    axis, freq = _pairs(case)
    outs = {}
    for side, h, x in _sides(case, s):
        x = x.double()
        if case["norm"] != "none":
            if case["norm"] == "layer":
                x = x - x.mean(-1, keepdim=True)
            x = x * (x.pow(2).sum(-1, keepdim=True) / case["D"] + 1e-6).rsqrt()
            x = x * (1.0 if s["w" + side] is None else s["w" + side].double()) + (0.0 if s["b" + side] is None else s["b" + side].double())
        y = x.clone()
        for i, (a, f) in enumerate(zip(axis, freq)):     # one pair after the other
            u, v = (i, i + len(axis)) if case["layout"] == "halves" else (2 * i, 2 * i + 1)
            t = s["pos"][..., a].double()[:, :, None] * f
            y[..., u] = x[..., u] * t.cos() - x[..., v] * t.sin()
            y[..., v] = x[..., u] * t.sin() + x[..., v] * t.cos()
        outs[side] = y if case["dst"] == "bshd" else y.transpose(1, 2)
    return outs


# ---- what is called ----------------------------------------------------------------------------------------------------
def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_adapters(case, g) if case["op"] == "adapters" else _prepare_heads(case, g)


def run(state):
    if own:
        from paper_2604_18117_b200 import binding as L
        stream = torch.cuda.current_stream().cuda_stream
        if state["op"] == "heads":
            return _own_heads(L, state, stream)
        L.lq_rowmap_set(state["map"].h, state["ids"].data_ptr(), state["M"], stream)       # once a step, for all of its linears
        return [_own_adapters(L, state, lin, stream) for lin in state["linears"]]
    return _plain_heads(state) if state["op"] == "heads" else [_plain_adapters(state, lin) for lin in state["linears"]]


def exact(case, seed):
    return _exact_adapters(case, seed) if case["op"] == "adapters" else _exact_heads(case, seed)


def work(case):
    """Adapters: X and Y0 in, Y out, the factors of the adapters in use once, each row's choice; both products.  Heads: Q and K in
    and out, positions; a norm and a rotation are some ten operations an entry."""
    nbytes = flops = 0
    if case["op"] == "adapters":
        M, ranks, req = case["M"], _ranks(case), _requests(case)
        n = len(req)
        rows = [(M * (i + 1) + n - 1) // n - (M * i + n - 1) // n for i in range(n)]       # of each request
        for K, N in _shapes(case):
            nbytes += 2 * M * K + 2 * M * N * (4 if case["out"] == "f32" else 2) + sum(2 * ranks[a] * (K + N) for a in set(req) if a >= 0)
            flops += sum(2 * m * ranks[a] * (K + N) for a, m in zip(req, rows) if a >= 0)
        nbytes += 4 * M
    else:
        n = case["B"] * case["S"] * (case["hq"] + case["hk"]) * case["D"]
        nbytes = n * sum(4 if case[k] == "f32" else 2 for k in ("fin", "fout")) + 4 * case["B"] * case["S"] * len(_ints(case["grid"]))
        flops = 10 * n
    return {"bytes": nbytes, "flops": flops}
