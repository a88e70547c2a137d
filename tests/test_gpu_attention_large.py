"""Attention where products are large: the whole range of finite queries and keys and of scales that the entry point takes.

Queries and keys here have products whose sums are whole numbers of 24 bits, so that what is expected is known exactly: what tells tokens
apart is not lost in the products' own rounding."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

from .test_gpu_kvcache import Cache

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def fill(c, lens, keys):
    """keys(s, n) -> [n][heads][D]; values are random."""
    import torch
    kv = [np.concatenate([keys(s, n) for s, n in enumerate(lens)]), np.concatenate([c.values(n) for n in lens])]
    turn = iter(kv)
    c.append(list(lens), make=lambda n: next(turn))
    for s, n in enumerate(lens):                           # (the cache holds them as they are)
        assert np.array_equal(c.held[0][s][:n], kv[0][sum(lens[:s]):sum(lens[:s + 1])])
    torch.cuda.synchronize()


def attend(c, ns, lens, q, scale, causal, uniform=False):
    import torch
    qd = torch.from_numpy(q.astype(np.float16)).cuda()
    assert np.array_equal(qd.double().cpu().numpy(), q)
    out = torch.full_like(qd, 7.0)
    B.lq_cache_attention(c.h, c.layer, c.batch(ns, lens, uniform), B.lq_attn(qd.data_ptr(), qd.stride()[:2], out.data_ptr(), out.stride()[:2], q.shape[1], scale, causal),
                         torch.cuda.current_stream().cuda_stream)
    got, at = out.double().cpu().numpy(), 0
    g = q.shape[1] // c.H
    for s, (n, t) in enumerate(zip(ns, lens)):
        for h in range(q.shape[1]):
            x = q[at:at + n, h] @ c.held[0][s][:t, h // g].T * scale
            v = c.held[1][s][:t, h // g]
            if causal:
                x = np.where(np.arange(t) <= t - n + np.arange(n)[:, None], x, -np.inf)
            x = x - x.max(1, keepdims=True)
            w = np.exp(x)
            total = w.sum(1, keepdims=True)
            want, near = w @ v / total, w @ np.abs(v) / total
            # A weight: rounded to a half, 2^-11 of it, or 2^-25 of the largest where it is that small; its exponent (a difference of two products, times the
            # scale, either within 4 u; the power within 8 u).  Where the maximum is followed late a reference may be rounded, to 2^-15.  Sums: 2 sqrt(n) + 64
            # roundings.
            far = np.where(np.isfinite(x) & (w > 0), -x, 0).max(1, keepdims=True)
            err = (2.0 ** -11 + 2.0 ** -14 + (8 * far + 16 + 2 * np.sqrt(t) + 64) * U) * near + (w > 0).sum(1, keepdims=True) * 2.0 ** -25 * np.abs(v).max() / total
            err += (np.abs(want) + err) * 2.0 ** -11 + 2.0 ** -25
            d = np.abs(got[at:at + n, h] - want) / err
            assert n == 0 or d.max() <= 1, (s, h, float(d.max()), np.unravel_index(d.argmax(), d.shape))
        at += n


# forms: single tokens; a long sequence over the grid; prompts; tiles of rows that are shared out; heads without tiles
FORMS = [([1, 1, 1], [40, 300, 2000], 64, 8, 2, True), ([1], [9001], 128, 8, 2, True), ([300, 70, 129], [300, 500, 129], 72, 4, 4, True),
         ([300, 300], [300, 700], 128, 4, 1, False), ([100], [4500], 64, 4, 1, True), ([60, 1], [100, 777], 256, 2, 1, True)]
IDS = ["tokens", "long", "prompts", "whole", "shared", "wide"]


@pytest.mark.parametrize("scale", [1.0, 2.0 ** 50, -(2.0 ** 50), 1.5e19])
@pytest.mark.parametrize("order", ["any", "rising"])
@pytest.mark.parametrize("ns,lens,D,hq,hk,causal", FORMS, ids=IDS)
def test_far_apart(ns, lens, D, hq, hk, causal, order, scale):
    """Products up to 2^30 and beyond 2^90: the largest has the weight, and tokens that share it share it."""
    c = Cache(D, hk, lens, 64)

    def keys(s, n):
        k = np.zeros((n, hk, D))
        k[..., 1] = 127 * 512.0
        code = c.rng.integers(1, 128, (n, hk)) if order == "any" else 1 + np.arange(n)[:, None] * 127 // n + np.zeros((1, hk))
        k[..., 0] = np.minimum(code, 127) * 512.0 * (1 if scale > 0 else -1)
        return k

    fill(c, lens, keys)
    q = np.zeros((sum(ns), hq, D))
    q[..., 0] = 8.0 * c.rng.integers(1025, 2048, (sum(ns), hq))
    attend(c, ns, lens, q, scale, causal)
    c.close()


@pytest.mark.parametrize("ns,lens,D,hq,hk,causal", FORMS, ids=IDS)
def test_far_out_but_close(ns, lens, D, hq, hk, causal):
    """Products around 2^31 that differ by a few units of the exponent, and grow along the sequence."""
    c = Cache(D, hk, lens, 64)

    def keys(s, n):
        k = np.zeros((n, hk, D))
        k[..., 2:4] = 64 * 512.0
        k[..., 0] = (c.rng.integers(-20, 0, (n, hk)) + 40 * (np.arange(n) // 100)[:, None].clip(max=2)) * 512.0
        k[..., 1] = 127 * 512.0
        return k

    fill(c, lens, keys)
    q = np.zeros((sum(ns), hq, D))
    q[..., 2:4] = 32768.0
    q[..., 0] = 2.0
    attend(c, ns, lens, q, 2.0 ** -11, causal)
    c.close()
