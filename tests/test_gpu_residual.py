"""The residual stream between two blocks, against the formula in 64 bits."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu

NORM = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
CODE = {"f16": B.OUT_F16, "f32": B.OUT_F32}
NP = {"f16": np.float16, "f32": np.float32}
U = 2.0 ** -24


def normed(x, ex, kind, eps):
    """(normed rows, how far an entry may be): x itself within ex.  Sums of C terms in a tree: within (C / 32 + 16) u of the sum of their magnitudes at most."""
    C = x.shape[1]
    k = (C / 32 + 16) * U
    if kind == "none":
        return x, ex
    m = 0.0
    if kind == "layer":
        m = x.mean(1, keepdims=True)
        ex = ex + (k + 2 * U) * np.abs(x).mean(1, keepdims=True) + ex.mean(1, keepdims=True) + U * np.abs(x - m)
    x = x - m
    r = 1 / np.sqrt(np.square(x).mean(1, keepdims=True) + eps)
    # the mean square moves by 2 x dx, and its root's inverse by half of that of itself, at most rms(dx) / rms(x)
    rel = k + 4 * U + np.sqrt(np.square(ex).mean(1, keepdims=True)) * r
    return x * r, ex * r + rel * np.abs(x * r)


def half(e, y, t):
    return e + (np.abs(y) + e) * (2.0 ** -11 if t == "f16" else U) + (2.0 ** -25 if t == "f16" else 0)


def run(M, C, Bn=1, after="none", norm="layer", mod="gcs", fx="f16", fy="f16", fh="f16", fm="f16", weights=True, factor=1.0, eps=1e-6, place="apart", y=True,
        want="xh", pad=0, flat=False):
    import torch
    rng = np.random.default_rng(M + C)
    dt = {"f16": torch.float16, "f32": torch.float32}
    xs = (rng.standard_normal((M, C)) * 3 + 2).astype(NP[fx])
    ys = (rng.standard_normal((M, C)) * np.exp(rng.standard_normal((M, 1)))).astype(NP[fy])
    if flat:
        xs[:], ys[:] = 3, 0
    put = lambda a, t: torch.nn.functional.pad(torch.from_numpy(a).cuda(), (0, pad), value=5.0).to(dt[t])
    xd, yd = put(xs, fx), put(ys, fy) if y else None
    vec = lambda: (1 + 0.3 * rng.standard_normal(C)).astype(np.float32)
    wa, w, b = (vec() if weights and c else None for c in (after != "none", norm != "none" and "h" in want, norm == "layer" and "h" in want))
    mods = (0.5 * rng.standard_normal((Bn, 6, C))).astype(NP[fm])
    md = torch.from_numpy(mods).cuda()
    wd = [None if v is None else torch.from_numpy(v).cuda() for v in (wa, w, b)]
    xo = xd if place == "in" else torch.full_like(xd, 9.0)
    hd = yd if place == "in" and y else torch.full((M, C + pad), 9.0, dtype=dt[fh], device="cuda")
    ptr = lambda v: None if v is None else v.data_ptr()
    g, sc, sh = (md[:, i].data_ptr() if c in mod else None for i, c in enumerate("gcs"))
    r = B.lq_residual(M, C, xd.data_ptr(), xo.data_ptr() if "x" in want else None, hd.data_ptr() if "h" in want else None, ptr(yd), Bn, NORM[after], ptr(wd[0]),
                      factor, g, NORM[norm], ptr(wd[1]), ptr(wd[2]), sc, sh, 6 * C, eps, CODE[fx], CODE[fy], CODE[fh], CODE[fm], (C + pad,) * 4)
    B.lq_residual_norm(r, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    rep = lambda i: np.repeat(mods[:, i].astype(np.float64), M // Bn, 0)
    x, e = xs.astype(np.float64), np.zeros((M, C))
    if y:
        v, ev = normed(ys.astype(np.float64), np.zeros((M, C)), after, eps)
        for f in ([wa.astype(np.float64)] if wa is not None else []) + ([rep(0)] if "g" in mod else []) + [np.float64(np.float32(factor))]:
            v = v * f
            ev = ev * np.abs(f) + U * np.abs(v)
        x = x + v
        e = ev + U * np.abs(x)
    if "x" in want:
        got = xo[:, :C].double().cpu().numpy()
        assert (np.abs(got - x) <= half(e, x, fx)).all()
        assert pad == 0 or (xo[:, C:] == (5 if place == "in" else 9)).all()
    if "h" in want:
        h, e = normed(x, e, norm, eps)
        for v, more in ((w, 0), (b, 1)):
            if v is not None:
                h = h + v if more else h * v
                e = (e if more else e * np.abs(v)) + U * np.abs(h)
        if "c" in mod:
            h = h * (1 + rep(1))
            e = e * np.abs(1 + rep(1)) + 2 * U * np.abs(h)
        if "s" in mod:
            h = h + rep(2)
            e = e + U * np.abs(h)
        got = hd[:, :C].double().cpu().numpy()
        far = np.abs(got - h) / half(e, h, fh)
        assert far.max() <= 1, float(far.max())


@pytest.mark.parametrize("C", [8, 72, 256, 264, 1000, 1024, 1032, 1152, 2048, 2240, 2312, 4096, 4104, 8192])
@pytest.mark.parametrize("M,Bn", [(1, 1), (6, 3), (9, 1)])
def test_sizes(M, Bn, C):
    run(M, C, Bn, after="rms")


@pytest.mark.parametrize("after", ["none", "rms", "layer"])
@pytest.mark.parametrize("norm", ["none", "rms", "layer"])
@pytest.mark.parametrize("types", [("f16", "f16", "f16", "f16"), ("f32", "f16", "f16", "f32"), ("f32", "f32", "f32", "f16"), ("f16", "f32", "f32", "f32")])
def test_norms_and_types(after, norm, types):
    for mod, weights in (("gcs", True), ("", True), ("g", False), ("cs", True), ("s", False), ("c", False)):
        run(34, 1152, 2, after, norm, mod, *types, weights=weights, factor=0.37)


@pytest.mark.parametrize("place", ["in", "apart"])
@pytest.mark.parametrize("C", [264, 4104])
def test_in_place_and_strides(place, C):
    run(50, C, 5, "layer", "rms", place=place, pad=16)
    run(50, C, 5, "layer", "rms", place=place, fx="f32", pad=8)


def test_parts():
    run(7, 320, y=False, mod="cs")
    run(7, 320, want="x", mod="g", norm="none")
    run(7, 320, want="h")
    run(7, 2240, y=False, mod="", want="h", norm="rms")


def test_many_rows():
    run(40000, 264, 8)
    run(6000, 2240, 3, "rms", "layer", fx="f32")


def test_rows_far_apart():
    """Rows behind 2^32 elements."""
    import torch
    C, far, M = 1152, (1 << 31) + 8, 3
    buf = torch.empty(2 * far + C, dtype=torch.float16, device="cuda")
    x = torch.as_strided(buf, (M, C), (far, 1))
    ref = torch.randn(M, C, device="cuda").half()
    x.copy_(ref)
    h = torch.empty(M, C, device="cuda")
    B.lq_residual_norm(B.lq_residual(M, C, x.data_ptr(), None, h.data_ptr(), norm=B.NORM_RMS, h_dtype=B.OUT_F32, strides=(far, C, C, C)),
                       torch.cuda.current_stream().cuda_stream)
    want, err = normed(ref.double().cpu().numpy(), np.zeros((M, C)), "rms", 1e-6)
    assert (np.abs(h.double().cpu().numpy() - want) <= err + U * np.abs(want)).all()


def test_rows_without_variance():
    run(5, 264, after="layer", norm="layer", flat=True, eps=1e-6)


def test_refusals():
    import torch
    x, y, z = (torch.zeros(8, 64, dtype=torch.float16, device="cuda") for _ in range(3))
    w = torch.zeros(64, device="cuda")
    X, Y, Z, W = (v.data_ptr() for v in (x, y, z, w))
    ok = dict(rows=8, features=64, x_ptr=X, x_out_ptr=X, h_ptr=Z, y_ptr=Y)
    make = lambda **k: B.lq_residual(**{**ok, **k})
    B.lq_residual_norm(make())
    for k, want in ((dict(x_ptr=0), 1), (dict(x_out_ptr=None, h_ptr=None), 1), (dict(rows=0), 1), (dict(features=0), 1), (dict(sequences=3), 1), (dict(sequences=0), 1),
                    (dict(after=3), 1), (dict(norm=-1), 1), (dict(x_dtype=2), 1), (dict(h_dtype=7), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1),
                    (dict(factor=float("inf")), 1), (dict(y_ptr=None, gate_ptr=W), 1), (dict(y_ptr=None, after=1), 1), (dict(after_weight_ptr=W), 1), (dict(weight_ptr=W), 1),
                    (dict(norm=1, bias_ptr=W), 1), (dict(h_ptr=None, norm=1), 1), (dict(h_ptr=None, shift_ptr=W), 1), (dict(features=60), 2), (dict(features=8200), 2),
                    (dict(x_ptr=X + 2), 1), (dict(strides=(60, 64, 64, 64)), 1), (dict(strides=(64, 64, 64, 1 << 40)), 2), (dict(device=77), 4),
                    (dict(h_ptr=X), 1), (dict(x_out_ptr=Y), 1), (dict(x_out_ptr=Z), 1), (dict(h_ptr=Y, h_dtype=1), 1), (dict(x_out_ptr=X, strides=(64, 64, 72, 64)), 1),
                    (dict(strides=(64, 64, 64, 32)), 1), (dict(norm=1, weight_ptr=Z), 1), (dict(gate_ptr=X), 1), (dict(mod_seq=4), 1)):
        with pytest.raises(B.LqError) as e:
            B.lq_residual_norm(make(**k))
        assert e.value.code == want, k
    torch.cuda.synchronize()
