"""Norms of queries and keys with the rotation by position, against the formulas in 64 bits."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu

NORMS = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}


def frequencies(dims, theta, shared):
    rot = sum(dims)
    axis = np.concatenate([np.full(d // 2, a, int) for a, d in enumerate(dims)]) if rot else np.zeros(0, int)
    if shared:
        return axis, theta ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    return axis, np.concatenate([theta ** (-2.0 * np.arange(d // 2) / max(d, 1)) for d in dims]) if rot else np.zeros(0)


def reference(x, w, b, norm, eps, axis, freq, halves, pos, f32_out):
    """x [B, S, H, D], pos [B, S, axes] -> (y in 64 bits, how far an element may be from it).  With u = 2^-24: a sum of D squares is within D u, so a
    normed value within (D / 2 + 8) u of itself (and, with a mean, that much of the mean magnitude, times the scale); cosine and sine are within 4 u of
    theirs; a turned value is two products and a sum."""
    u, D = 2.0 ** -24, x.shape[-1]
    x = x.astype(np.float64)
    err = np.zeros_like(x)
    if norm != "none":
        w64 = np.ones(D) if w is None else w.astype(np.float64)
        m = x.mean(-1, keepdims=True) if norm == "layer" else 0.0
        rstd = 1 / np.sqrt(np.square(x - m).mean(-1, keepdims=True) + eps)
        if norm == "layer":
            err = 2 * D * u * np.abs(x).mean(-1, keepdims=True) * rstd * np.abs(w64) * np.ones_like(x)
            # (the mean's error moves the variance only in second order)
        x = (x - m) * rstd * w64
        err = err + (D / 2 + 8) * u * np.abs(x)
        if b is not None:
            x = x + b
            err = err + u * np.abs(x)
    P = freq.size
    y, e = x.copy(), err.copy()
    if P:
        t = pos.astype(np.float64)[..., axis] * freq
        c, s = np.cos(t)[:, :, None], np.sin(t)[:, :, None]
        lo = slice(0, P) if halves else slice(0, 2 * P, 2)
        hi = slice(P, 2 * P) if halves else slice(1, 2 * P, 2)
        y[..., lo], y[..., hi] = x[..., lo] * c - x[..., hi] * s, x[..., hi] * c + x[..., lo] * s
        both = np.abs(x[..., lo]) + np.abs(x[..., hi])
        # the reference's own angle: 2^-52 of pos * freq
        off = (8 * u + 2.0 ** -51 * np.abs(t)[:, :, None]) * both + err[..., lo] + err[..., hi]
        e[..., lo] = e[..., hi] = off
    return y, e + (np.abs(y) + e) * (u if f32_out else 2.0 ** -11) + (0 if f32_out else 2.0 ** -25)


class Case:
    def __init__(self, Bn, S, hq, hk, D, norm, dims, halves=False, shared=False, theta=10000.0, far=1000, fin="f16", fout="f16",
                 weight=True, in_place=False, bhsd=False, seed=0, freq=None, axis=None):
        import torch
        rng = np.random.default_rng(seed + D + S)
        self.norm, self.halves, self.fout = norm, halves, fout
        ti, to = (torch.float32 if f == "f32" else torch.float16 for f in (fin, fout))
        hv = 1                                             # a head of other values behind the keys
        x = rng.standard_normal((Bn, S, hq + hk + hv, D)).astype(np.float32) * np.exp(rng.standard_normal((1, 1, hq + hk + hv, 1)))
        self.x = x.astype(np.float32 if fin == "f32" else np.float16)
        self.pos = rng.integers(-far, far + 1, (Bn, S, max(1, len(dims)))).astype(np.int32)
        self.axis, self.freq = frequencies(dims, theta, shared)
        cfg = B.lq_rope_config_default(dims, theta=theta, halves=halves, shared=shared)
        if freq is not None:
            self.freq = freq
        if axis is not None:
            self.axis = axis
        self.rope = B.lq_rope_create(cfg, 0, freq, axis)
        vec = lambda: (1 + 0.3 * rng.standard_normal(D)).astype(np.float32)
        self.w = [vec() if weight and norm != "none" else None for _ in range(2)]
        self.b = [vec() if weight and norm == "layer" else None for _ in range(2)]
        put = lambda a: None if a is None else torch.from_numpy(a).cuda()
        self.wd, self.bd = [put(v) for v in self.w], [put(v) for v in self.b]
        rows = torch.from_numpy(self.x).cuda().to(ti)
        posd = torch.from_numpy(self.pos).cuda()
        sides, self.out, at = [], [], 0
        for i, h in enumerate((hq, hk)):
            src = rows[:, :, at:at + h]
            at += h
            if h == 0:
                sides.append(None)
                self.out.append(None)
                continue
            if in_place:
                dst, strides = src, src.stride()[:3]
            elif bhsd:
                dst = torch.full((Bn, h, S, D), 9.0, dtype=to, device="cuda")
                strides = [dst.stride(0), dst.stride(2), dst.stride(1)]
            else:
                dst = torch.full((Bn, S, h, D), 9.0, dtype=to, device="cuda")
                strides = dst.stride()[:3]
            self.out.append(dst)
            sides.append(B.lq_heads(src.data_ptr(), src.stride()[:3], dst.data_ptr(), strides, h,
                                    None if self.wd[i] is None else self.wd[i].data_ptr(), None if self.bd[i] is None else self.bd[i].data_ptr()))
        code = {"f16": B.OUT_F16, "f32": B.OUT_F32}
        self.kept = [rows, posd]
        self.call = lambda st: B.lq_qk_norm_rope(sides[0], sides[1], D, Bn, S, NORMS[norm], 1e-6, self.rope, posd.data_ptr() if dims else None,
                                                 code[fin], code[fout], st)
        self.h, self.rows, self.in_place, self.bhsd = (hq, hk), rows, in_place, bhsd

    def check(self):
        at = 0
        for i, h in enumerate(self.h):
            if h:
                y = self.out[i].float().cpu().numpy()
                y = y.transpose(0, 2, 1, 3) if self.bhsd and not self.in_place else y
                ref, bound = reference(self.x[:, :, at:at + h], self.w[i], self.b[i], self.norm, 1e-6, self.axis, self.freq, self.halves, self.pos,
                                       self.fout == "f32")
                over = np.abs(y - ref) - bound
                assert over.max() <= 0, ("qk"[i], over.max(), np.unravel_index(over.argmax(), y.shape))
            at += h
        assert np.array_equal(self.rows[:, :, at:].cpu().numpy(), self.x[:, :, at:])       # what lies beside the heads stays
        B.lq_rope_free(self.rope)

    def run(self):
        import torch
        self.call(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        self.check()


@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("D,dims", [(8, (8,)), (32, (32,)), (40, (16,)), (64, (24, 40)), (72, (72,)), (72, (36, 36)), (80, ()), (96, (32, 32, 32)),
                                    (112, (96,)), (128, (44, 42, 42)), (160, (40, 40, 40, 40)), (248, (8,)), (256, (256,))])
def test_head_sizes_against_64_bits(norm, halves, D, dims):
    Case(2, 37, 3, 2, D, norm, dims, halves=halves).run()


@pytest.mark.parametrize("fin,fout", [("f16", "f16"), ("f16", "f32"), ("f32", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("Bn,S,hq,hk", [(1, 1, 1, 0), (1, 1, 0, 3), (1, 1, 16, 16), (5, 1, 32, 8), (1, 513, 1, 1), (3, 455, 20, 5), (2, 300, 64, 1)])
@pytest.mark.parametrize("D,halves", [(72, True), (128, False), (128, True)])
def test_rows_heads_and_types(fin, fout, Bn, S, hq, hk, D, halves):
    Case(Bn, S, hq, hk, D, "rms", (D - 8,), halves=halves, fin=fin, fout=fout, bhsd=S % 2 == 1).run()


# Heads of 64, 72, 112 and 128 entries, turned as a whole or not at all, have instances of their own under an RMS norm; the others have the
# general one.  Rows enough for two a block (1776 and more on 148 SMs, the last block with one), heads enough for a warp to take more steps
# than it has loads in flight (three: eight, three, two, four heads a step, and one or more of the general form).
LONG = {64: 40, 72: 16, 112: 10, 128: 20, 80: 13, 96: 15, 160: 7, 256: 5}


@pytest.mark.parametrize("fin,fout", [("f16", "f16"), ("f16", "f32"), ("f32", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("turned", ["none", "pairs", "halves"])
@pytest.mark.parametrize("D", [64, 72, 112, 128])
def test_long_walks_of_the_instances_by_size(D, turned, fin, fout):
    dims = () if turned == "none" else (D - 24, 24) if turned == "pairs" else (D,)
    Case(1, 1777, LONG[D], LONG[D], D, "rms", dims, halves=turned == "halves", fin=fin, fout=fout).run()
    Case(3, 7, LONG[D], 3, D, "rms", dims, halves=turned == "halves", fin=fin, fout=fout, bhsd=True, weight=False).run()


@pytest.mark.parametrize("fin,fout", [("f16", "f16"), ("f16", "f32"), ("f32", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("D,dims,norm", [(64, (64,), "layer"), (72, (40,), "rms"), (80, (80,), "rms"), (96, (64,), "layer"), (128, (128,), "none"),
                                         (160, (160,), "none"), (256, (), "layer"), (112, (112,), "layer")])
def test_long_walks_of_the_general_instance(D, dims, norm, fin, fout):
    Case(1, 1777, LONG[D], LONG[D], D, norm, dims, halves=D % 64 == 0, fin=fin, fout=fout).run()
    Case(2, 889, LONG[D] + 5, LONG[D], D, norm, dims, halves=D % 64 == 0, fin=fin, fout=fout, in_place=fin == fout).run()


@pytest.mark.parametrize("fin", ["f16", "f32"])
@pytest.mark.parametrize("halves", [False, True])
def test_in_place(fin, halves):
    Case(2, 130, 4, 4, 72, "rms", (24, 24, 24), halves=halves, fin=fin, fout=fin, in_place=True).run()
    Case(1, 77, 6, 2, 64, "layer", (32,), halves=halves, fin=fin, fout=fin, in_place=True, weight=False).run()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("halves", [False, True])
def test_axes_share_or_own_their_frequencies(shared, halves):
    Case(2, 60, 2, 1, 128, "none", (32, 48, 48), halves=halves, shared=shared, theta=1e6, fin="f32", fout="f32").run()
    Case(1, 9, 2, 1, 64, "rms", (0, 64, 0, 0), halves=halves, shared=shared).run()


def test_angles_of_far_positions_are_exact():
    """2^31 - 1 positions away an angle in 32 bits would be off by hundreds of radians."""
    for far in (10 ** 6, 2 ** 31 - 1):
        Case(1, 200, 1, 1, 64, "none", (64,), far=far, fin="f32", fout="f32").run()


def test_frequencies_and_axes_of_the_caller():
    rng = np.random.default_rng(0)
    freq = np.concatenate([[0.0, 1.0, np.pi, -0.5, 2 * np.pi, 100.0], rng.random(26)])
    Case(1, 50, 2, 2, 64, "none", (64, 0, 0), freq=freq, axis=rng.integers(0, 3, 32), fin="f32", fout="f32").run()


def test_fast_frequencies_at_far_positions():
    """Many turns a position, up to 2^31 positions away, against angles from whole numbers of 400 bits: the fraction of a turn that is kept is
    right whatever the whole turns before it."""
    import torch
    from fractions import Fraction
    from tests.test_turns_host import pi
    freq = np.array([100.0, -12345.678, 1e6, 3.7e9, -2.0 ** 40 - 0.5, 1e15 + 0.125, 2.0 ** 63, 6.0])
    pos = np.array([1, -1, 12345, 10 ** 8 + 1, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1], np.int32)
    two_pi = 2 * pi()
    t = np.array([[float((int(p) * Fraction(float(f)) / two_pi % 1 + Fraction(1, 2)) % 1 - Fraction(1, 2)) for f in freq] for p in pos]) * 2 * np.pi
    S, D = pos.size, 16
    rng = np.random.default_rng(3)
    x = rng.standard_normal((S, 1, D)).astype(np.float32)
    rope = B.lq_rope_create(B.lq_rope_config_default([D]), 0, freq)
    xd, pd, out = torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda(), torch.zeros(S, 1, D, device="cuda")
    side = B.lq_heads(xd.data_ptr(), (S * D, D, D), out.data_ptr(), (S * D, D, D), 1)
    B.lq_qk_norm_rope(side, None, D, 1, S, B.NORM_NONE, 0.0, rope, pd.data_ptr(), B.OUT_F32, B.OUT_F32, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    B.lq_rope_free(rope)
    u, v = x[:, 0, 0::2].astype(np.float64), x[:, 0, 1::2].astype(np.float64)
    y = out.cpu().numpy()[:, 0].astype(np.float64)
    # cosine and sine within 4 * 2^-24 of theirs, two products and a sum, a rounding: as in reference()
    bound = 10 * 2.0 ** -24 * (np.abs(u) + np.abs(v))
    assert (np.abs(y[:, 0::2] - (u * np.cos(t) - v * np.sin(t))) <= bound).all()
    assert (np.abs(y[:, 1::2] - (v * np.cos(t) + u * np.sin(t))) <= bound).all()


def test_angles_err_to_both_sides():
    """The mean of a million angles' errors.  One is off by 2.3e-8 radians (root mean square: floats near an eighth of a turn), their mean so by
    3e-11 and, as those of one position are not independent, a few times that.  Angles cut to 32 bits of a turn are 2 pi / 2^33 = 7.3e-10
    short on average; half of that is the limit."""
    import torch
    from fractions import Fraction
    from tests.test_turns_host import pi
    rng = np.random.default_rng(0)
    S, P = 8192, 128
    freq, pos = rng.uniform(0.1, 3.0, P), rng.integers(-2 ** 20, 2 ** 20, S).astype(np.int32)
    two_pi = 2 * pi()
    turn = np.array([round(Fraction(float(f)) / two_pi * 2 ** 64) % 2 ** 64 for f in freq], np.uint64)
    t = (turn[None] * pos.astype(np.int64).astype(np.uint64)[:, None]).astype(np.int64) * 2.0 ** -64 * 2 * np.pi
    x = np.zeros((S, 2 * P), np.float32)
    x[:, 0::2] = 1
    rope = B.lq_rope_create(B.lq_rope_config_default([2 * P]), 0, freq)
    xd, pd = torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda()
    out = torch.zeros_like(xd)
    side = B.lq_heads(xd.data_ptr(), (0, 2 * P, 0), out.data_ptr(), (0, 2 * P, 0), 1)
    B.lq_qk_norm_rope(side, None, 2 * P, 1, S, B.NORM_NONE, 0.0, rope, pd.data_ptr(), B.OUT_F32, B.OUT_F32, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    B.lq_rope_free(rope)
    y = out.cpu().numpy().astype(np.float64)
    err = y[:, 1::2] * np.cos(t) - y[:, 0::2] * np.sin(t)
    assert np.abs(err).max() <= 8 * 2.0 ** -24 and abs(err.mean()) <= 2 * np.pi * 2.0 ** -34, (np.abs(err).max(), err.mean())


def test_zero_heads_and_large_values():
    """A head of zeros stays zero; fp32 entries whose squares are large or tiny."""
    import torch
    c = Case(1, 40, 2, 2, 72, "rms", (72,), fin="f32", fout="f32")
    c.x[0, 3, 0] = 0
    c.x[0, 4, 1] *= 1e15
    c.x[0, 5, 2] *= 1e-15
    c.rows.copy_(torch.from_numpy(c.x))
    c.run()
    assert not c.out[0][0, 3, 0].any()


def test_a_nan_stays_in_its_head():
    import torch
    for D in (72, 128):
        c = Case(1, 20, 3, 1, D, "rms", (D,), halves=True)
        c.rows[0, 5, 1, 7] = float("nan")
        c.call(torch.cuda.current_stream().cuda_stream)
        bad = ~torch.isfinite(c.out[0].float()).all(-1)
        assert bad[0, 5, 1] and bad.sum() == 1 and torch.isfinite(c.out[1]).all()
        B.lq_rope_free(c.rope)


def test_captured_and_replayed_on_another_stream():
    import torch
    c = Case(2, 100, 4, 2, 72, "rms", (36, 36))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.call(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.call(torch.cuda.current_stream().cuda_stream)
    c.x = (c.x * 0.5 + 1).astype(np.float16)
    c.pos[:] += 17
    c.kept[0].copy_(torch.from_numpy(c.x))
    c.kept[1].copy_(torch.from_numpy(c.pos))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    c.check()


def test_refusals():
    import torch
    x = torch.zeros(1 << 14, dtype=torch.float16, device="cuda")
    P = x.data_ptr()
    w = torch.ones(64, device="cuda").data_ptr()
    rope, none = B.lq_rope_create(B.lq_rope_config_default([64]), 0), B.lq_rope_create(B.lq_rope_config_default([]), 0)
    pos = torch.zeros(64, dtype=torch.int32, device="cuda").data_ptr()
    good = dict(in_ptr=P, in_strides=(0, 128, 64), out_ptr=P + 16384, out_strides=(0, 128, 64), heads=2)

    def code(side=None, q=True, D=64, Bn=1, S=4, norm=B.NORM_RMS, eps=1e-6, r=rope, at=pos, fin=0, fout=0):
        h = B.lq_heads(**{**good, **(side or {})})
        try:
            B.lq_qk_norm_rope(h if q else None, None, D, Bn, S, norm, eps, r, at, fin, fout, 0)
        except B.LqError as e:
            return e.code
        return 0

    assert code() == 0 and code(r=none, at=None) == 0
    assert code(dict(in_strides=(3, 128, 64))) == 0                                       # one sequence: its stride means nothing
    for side in (dict(in_ptr=None), dict(out_ptr=None), dict(in_ptr=P + 8), dict(out_ptr=P + 8), dict(heads=0), dict(in_strides=(0, 124, 64)),
                 dict(out_strides=(0, 128, 60)), dict(out_strides=(0, 0, 64)), dict(out_strides=(0, 128, 0)), dict(bias_ptr=w), dict(weight_ptr=w + 4)):
        assert code(side) == 1, side
    assert code(dict(weight_ptr=w), norm=B.NORM_NONE) == 1 and code(dict(weight_ptr=w, bias_ptr=w), norm=B.NORM_LAYER) == 0
    assert code(q=False) == 1 and code(Bn=0) == 1 and code(S=0) == 1 and code(norm=3) == 1 and code(eps=-1.0) == 1 and code(eps=float("nan")) == 1
    assert code(fin=2) == 1 and code(fout=2) == 1 and code(at=None) == 1 and code(at=pos + 2) == 1 and code(D=0) == 1
    assert code(D=60) == 2 and code(D=264) == 2 and code(dict(heads=5000)) == 2
    assert code(D=56, side=dict(in_strides=(0, 128, 56), out_strides=(0, 128, 56))) == 1   # fewer entries than are rotated
    torch.cuda.synchronize()
    B.lq_rope_free(rope)
    B.lq_rope_free(none)


def test_outputs_on_one_place_and_other_ways_in_place_are_refused():
    import torch
    x = torch.zeros(1 << 14, dtype=torch.float16, device="cuda")
    P = x.data_ptr()
    none = B.lq_rope_create(B.lq_rope_config_default([]), 0)

    def code(q, k=None, fin=0, fout=0, Bn=2):
        try:
            B.lq_qk_norm_rope(B.lq_heads(*q), B.lq_heads(*k) if k else None, 64, Bn, 4, B.NORM_RMS, 1e-6, none, None, fin, fout, 0)
        except B.LqError as e:
            return e.code
        return 0

    good, far = (512, 128, 64), P + 16384
    assert code((P, good, far, good, 2)) == 0 and code((P, good, P, good, 2)) == 0 and code((P, good, far, (64, 256, 128), 2), Bn=1) == 0
    for bad in ((512, 128, 56), (512, 128, -56), (512, 56, 128), (56, 128, 64)):
        assert code((P, good, far, bad, 2)) == 1, bad
    assert code((P, good, P, (512, 128, 72), 2)) == 1 and code((P, good, P, good, 2), fout=1) == 1 and code((P, good, P, good, 2), fin=1) == 1
    assert code((P, good, far, good, 1), (P + 128, good, far, good, 1)) == 1
    torch.cuda.synchronize()
    B.lq_rope_free(none)


def test_every_output_has_a_place_of_its_own_apart_from_the_inputs():
    """Dimensions that run through one another, a side's output on the other's input, on its own input shifted, on weights or positions: refused,
    and nothing is written.  The same without a shared place: taken."""
    import torch
    x = torch.zeros(1 << 15, dtype=torch.float16, device="cuda")
    x[:] = torch.arange(1 << 15, device="cuda") % 100
    before = x.clone()
    P, far = x.data_ptr(), x.data_ptr() + 32768
    rope = B.lq_rope_create(B.lq_rope_config_default([64]), 0)
    pos = torch.zeros(8, dtype=torch.int32, device="cuda").data_ptr()

    def code(q, k=None, Bn=2, at=pos, fin=0, fout=0):
        try:
            B.lq_qk_norm_rope(B.lq_heads(*q), B.lq_heads(*k) if k else None, 64, Bn, 4, B.NORM_RMS, 1e-6, rope, at, fin, fout, 0)
        except B.LqError as e:
            return e.code
        return 0

    s = (512, 128, 64)
    for bad in ((512, 64, 64), (512, 128, 128), (128, 128, 64), (256, 128, 64), (512, 128, -128), (512, 128, 256)):
        assert code((P, s, far, bad, 2)) == 1, bad
    for q, k in (((P, s, far, s, 2), (P + 2048, s, P, s, 2)),                    # keys onto what queries are read from
                 ((P, s, P + 2048, s, 2), (P + 2048, s, far, s, 2)),             # queries onto what keys are read from
                 ((P, s, far, s, 2), (P + 2048, s, far + 128, s, 2)),            # the keys' first head on the queries' second
                 ((P, s, far, (512, 128, 64), 1), (P + 2048, s, far + 64, s, 1)),
                 ((P, s, P, s, 2), (P + 128, s, P + 128, s, 1))):                # in place, and one head of both sides
        assert code(q, k) == 1, (q, k)
    assert code((P, s, P + 128, s, 1)) == 0 and code((P, s, P + 16, s, 1)) == 1 and code((P, s, P + 128, s, 2)) == 1
    assert code((P, s, far, s, 2, far + 1024)) == 1 and code((P, s, far, s, 2), at=far + 4) == 1
    assert code((P, s, far, s, 2), fout=1) == 0 and code((P, s, far - 2560, s, 2), fout=1) == 0 and code((P, s, P + 1024, s, 2), fout=1) == 1
    torch.cuda.synchronize()
    x.copy_(before)
    torch.cuda.synchronize()
    for q, k in (((P, s, far, s, 2), (P + 2048, s, P, s, 2)), ((P, s, P, s, 2), (P + 128, s, P + 128, s, 1))):
        assert code(q, k) == 1
    torch.cuda.synchronize()
    assert torch.equal(x, before)
    assert code((P, s, P, s, 1), (P + 128, s, P + 128, s, 1)) == 0               # in place, side by side in a row
    assert code((P, s, far, (1024, 256, 128), 2), (P + 2048, s, far + 128, (1024, 256, 128), 2)) == 0      # a query beside its key
    assert code((P, s, far, (0, 512, 384), 2), Bn=1) == 0                        # woven, every place once
    torch.cuda.synchronize()
    B.lq_rope_free(rope)


@pytest.mark.parametrize("norm", ["none", "rms"])
def test_strides_backwards_and_far_apart(norm):
    """Rows in the opposite order, heads too, and sequences of outputs 2^30 elements and more apart."""
    import torch
    rng = np.random.default_rng(11)
    Bn, S, h, D = 4, 5, 3, 64
    x = rng.standard_normal((Bn, S, h, D)).astype(np.float16)
    pos = rng.integers(0, 1000, (Bn, S, 1)).astype(np.int32)
    axis, freq = frequencies([D], 10000.0, False)
    rope = B.lq_rope_create(B.lq_rope_config_default([D]), 0)
    xd, pd = torch.from_numpy(x).cuda(), torch.from_numpy(pos).cuda()
    apart = 1 << 30
    out = torch.empty(3 * apart + S * h * D, dtype=torch.float16, device="cuda")
    last = (S - 1) * h * D + (h - 1) * D                   # the place of the first row's first head
    side = B.lq_heads(xd.data_ptr(), (S * h * D, h * D, D), out.data_ptr() + 2 * last, (apart, -h * D, -D), h)
    B.lq_qk_norm_rope(side, None, D, Bn, S, NORMS[norm], 1e-6, rope, pd.data_ptr(), B.OUT_F16, B.OUT_F16, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    ref, bound = reference(x, None, None, norm, 1e-6, axis, freq, False, pos, False)
    for b in range(Bn):
        got = out[b * apart:b * apart + S * h * D].view(S, h, D).flip(0, 1).float().cpu().numpy()
        assert (np.abs(got - ref[b]) <= bound[b]).all(), b
    B.lq_rope_free(rope)


def test_positions_are_ignored_without_axes():
    import torch
    x = torch.ones(4 * 64, dtype=torch.float16, device="cuda")
    side = B.lq_heads(x.data_ptr(), (0, 64, 0), x.data_ptr(), (0, 64, 0), 1)
    for dims in ([], [0, 0]):
        rope = B.lq_rope_create(B.lq_rope_config_default(dims), 0)
        for pos in (None, 1, x.data_ptr() + 2):
            B.lq_qk_norm_rope(side, None, 64, 1, 4, B.NORM_RMS, 0.0, rope, pos, B.OUT_F16, B.OUT_F16, 0)
        torch.cuda.synchronize()
        B.lq_rope_free(rope)
    assert (x == 1).all()


@pytest.mark.parametrize("sequences", [1, 2])
def test_the_longest_strides(sequences):
    """The largest multiple of eight below 2^31, of rows and of sequences; the next one is refused."""
    import torch
    rng = np.random.default_rng(2)
    D, apart = 8, 2 ** 31 - 8
    x, y = (torch.empty(apart + D, dtype=torch.float16, device="cuda") for _ in range(2))
    rows = rng.standard_normal((2, D)).astype(np.float16)
    x[:D], x[apart:] = torch.from_numpy(rows[0]).cuda(), torch.from_numpy(rows[1]).cuda()
    rope = B.lq_rope_create(B.lq_rope_config_default([]), 0)
    S = 2 // sequences

    def call(step, back=1):
        at = [t.data_ptr() + (2 * apart if back < 0 else 0) for t in (x, y)]
        strides = (back * step, back * step, 0)
        side = B.lq_heads(at[0], strides, at[1], strides, 1)
        B.lq_qk_norm_rope(side, None, D, sequences, S, B.NORM_RMS, 1e-6, rope, None, B.OUT_F16, B.OUT_F16, torch.cuda.current_stream().cuda_stream)

    ref, bound = reference(rows[:, None, None], None, None, "rms", 1e-6, np.zeros(0, int), np.zeros(0), False, None, False)
    for back in (1, -1):
        y[:D] = y[apart:] = 9
        call(apart, back)
        torch.cuda.synchronize()
        got = torch.stack([y[:D], y[apart:]]).float().cpu().numpy()
        assert (np.abs(got - ref[:, 0, 0]) <= bound[:, 0, 0]).all(), back
        with pytest.raises(B.LqError) as e:
            call(apart + 8, back)
        assert e.value.code == 2
    B.lq_rope_free(rope)


def test_the_most_heads_of_the_longest():
    for norm in ("rms", "layer"):
        Case(1, 1, 4095, 7, 256, norm, (256,)).run()
        Case(1, 3, 1, 4096, 8, norm, (8,), halves=True).run()


def test_the_most_rows():
    """2^31 - 1 rows of one head of eight entries, in place."""
    import torch
    n, D = 2 ** 31 - 1, 8
    if torch.cuda.mem_get_info()[0] < 44e9:
        pytest.skip("the rows alone are 34 GB")
    x = torch.full((n, D), 3.0, dtype=torch.float16, device="cuda")
    look = torch.tensor([0, 1, 2, n // 2, n - 3, n - 2, n - 1], device="cuda")
    rng = np.random.default_rng(0)
    rows = rng.standard_normal((look.numel(), D)).astype(np.float16)
    x[look] = torch.from_numpy(rows).cuda()
    rope = B.lq_rope_create(B.lq_rope_config_default([]), 0)
    side = B.lq_heads(x.data_ptr(), (0, D, 0), x.data_ptr(), (0, D, 0), 1)
    B.lq_qk_norm_rope(side, None, D, 1, n, B.NORM_RMS, 0.0, rope, None, B.OUT_F16, B.OUT_F16, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    B.lq_rope_free(rope)
    ref, bound = reference(rows[None, :, None], None, None, "rms", 0.0, np.zeros(0, int), np.zeros(0), False, None, False)
    assert (np.abs(x[look].float().cpu().numpy() - ref[0, :, 0]) <= bound[0, :, 0]).all()
    x[look] = 1.0                                          # the others: 3 / sqrt(9) within a rounding
    for part in x.view(-1).split(1 << 28):
        lo, hi = torch.aminmax(part)
        assert abs(float(lo) - 1) <= 2.0 ** -11 and abs(float(hi) - 1) <= 2.0 ** -11
    del x, part
    torch.cuda.empty_cache()
