"""The 8-bit cache of keys and values, what is written and read, and attention over it, against the definitions in 64 bits."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu

E_MIN, E_MAX, BLOCK = -20, 9, 32


def exponent(top):
    e = E_MIN
    while e < E_MAX and 127 * 2.0 ** e < top:
        e += 1
    return e


def write(held, exps, x, at):
    """Tokens at .. at + len(x) - 1 of held [tokens][heads][D]; exps {(block, head): exponent}."""
    for h in range(x.shape[1]):
        done = 0
        while done < len(x):
            t = at + done
            n = min(len(x) - done, BLOCK - t % BLOCK)
            new, key, first = x[done:done + n, h], (t // BLOCK, h), t // BLOCK * BLOCK
            need = exponent(np.abs(new).max())
            e = max(need, exps[key]) if t % BLOCK else need
            if t % BLOCK and e > exps[key]:
                old = held[first:t, h] / 2.0 ** exps[key]
                held[first:t, h] = np.round(old / 2.0 ** (e - exps[key])) * 2.0 ** e
            held[t:t + n, h] = np.clip(np.round(new / 2.0 ** e), -127, 127) * 2.0 ** e
            exps[key] = e
            done += n


class Cache:
    """A cache and its sequences, beside what it should hold."""

    def __init__(self, D, heads, lens, page=32, layers=1, layer=0, seed=0, spare=2):
        import torch
        self.D, self.H, self.page, self.layer = D, heads, page, layer
        self.rng = np.random.default_rng(seed + D + 7 * heads)
        self.B = len(lens)
        counts = [-(-n // page) for n in lens]
        self.stride = max(1, max(counts))
        n_pages = sum(counts) + spare
        order = self.rng.permutation(n_pages)
        self.pages = np.full((self.B, self.stride), -1, np.int32)
        at = 0
        for s, c in enumerate(counts):
            self.pages[s, :c] = order[at:at + c]
            at += c
        self.h = B.lq_kvcache_create(layers, n_pages, page, heads, D)
        self.pages_d = torch.from_numpy(self.pages).cuda()
        self.len = [0] * self.B
        self.held = [[np.zeros((n + 1, heads, D)) for n in lens] for _ in "kv"]
        self.exps = [[{} for _ in lens] for _ in "kv"]
        self.keep = []

    def batch(self, ns, lens, uniform=False, behind=0):
        import torch
        start = np.concatenate([[0], np.cumsum(ns)]).astype(np.int32)
        sd, ld = torch.from_numpy(start).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.keep = [sd, ld]
        return B.lq_kvbatch(self.B, int(start[-1]) + behind, ld.data_ptr(), self.pages_d.data_ptr(), self.stride, None if uniform else sd.data_ptr())

    def values(self, n):
        x = self.rng.standard_normal((n, self.H, self.D)) * np.exp(self.rng.standard_normal((1, self.H, 1)))
        return x * np.exp2(self.rng.integers(-3, 4, (n, 1, 1)))        # tokens of different size: exponents grow

    def append(self, ns, dtype="f16", uniform=False, make=None, stream=None):
        """ns new tokens of each sequence, K and V in rows of [V heads, K heads, others]."""
        import torch
        t = torch.float16 if dtype == "f16" else torch.float32
        rows = sum(ns)
        kv = [(make or self.values)(rows).astype(np.float16 if dtype == "f16" else np.float32) for _ in "kv"]
        buf = torch.zeros(rows + 1, 2 * self.H + 1, self.D, dtype=t, device="cuda")
        buf[:rows, self.H:2 * self.H] = torch.from_numpy(kv[0]).cuda()
        buf[:rows, :self.H] = torch.from_numpy(kv[1]).cuda()
        self.len = [a + n for a, n in zip(self.len, ns)]
        b = self.batch(ns, self.len, uniform)
        row = (2 * self.H + 1) * self.D
        r = B.lq_kvrows(buf[:, self.H:].data_ptr(), (0, row, self.D), buf.data_ptr(), (0, row, self.D))
        B.lq_kvcache_append(self.h, self.layer, b, r, B.OUT_F16 if dtype == "f16" else B.OUT_F32, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for side in range(2):
            at = 0
            for s, n in enumerate(ns):
                if n:
                    write(self.held[side][s], self.exps[side][s], kv[side][at:at + n].astype(np.float64), self.len[s] - n)
                at += n

    def read(self, begin=None, most=None, dtype="f32"):
        import torch
        t = torch.float16 if dtype == "f16" else torch.float32
        most = most or max(1, max(self.len))
        out = torch.full((2, self.B, self.H, most, self.D), 77.0, dtype=t, device="cuda")       # heads apart in memory
        b = self.batch([0] * self.B, self.len)
        bd = None if begin is None else torch.tensor(begin, dtype=torch.int32, device="cuda")
        st = (out.stride(1), out.stride(3), out.stride(2))
        B.lq_kvcache_read(self.h, self.layer, b, None if bd is None else bd.data_ptr(), most, B.lq_kvrows(out[0].data_ptr(), st, out[1].data_ptr(), st),
                          B.OUT_F16 if dtype == "f16" else B.OUT_F32, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return out.float().cpu().numpy()

    def check(self, begin=None, most=None, dtype="f32"):
        got = self.read(begin, most, dtype)
        for side in range(2):
            for s in range(self.B):
                b = 0 if begin is None else begin[s]
                want = self.held[side][s][b:self.len[s]][: got.shape[3]].transpose(1, 0, 2)
                n = want.shape[1]
                assert np.array_equal(got[side, s, :, :n], want), (side, s)
                assert (got[side, s, :, n:] == 77).all()

    def close(self):
        assert B.lq_get_device_status(0) == (0, 0)
        B.lq_kvcache_free(self.h)


@pytest.mark.parametrize("D,heads,page,dtype", [(8, 1, 32, "f16"), (16, 3, 64, "f32"), (64, 2, 32, "f16"), (72, 5, 96, "f16"), (80, 1, 32, "f32"),
                                                (96, 2, 64, "f16"), (112, 4, 128, "f32"), (128, 8, 64, "f16"), (160, 2, 32, "f16"), (256, 2, 256, "f32")])
def test_what_is_written_is_read(D, heads, page, dtype):
    c = Cache(D, heads, [200, 70, 33, 140], page)
    for ns in ([1, 33, 0, 64], [1, 0, 1, 1], [30, 1, 31, 1], [1, 1, 0, 31], [5, 2, 1, 1], [100, 33, 0, 40], [1, 0, 0, 2]):
        c.append(ns, dtype)
        c.check()
    c.check(begin=[32, 5, 33, 64])
    c.check(begin=[64, 70, 0, 1], most=40)
    c.check(dtype="f16")
    c.close()


def test_one_row_of_every_sequence():
    """The form without row_start; a token at a time from the first on, over more than a block."""
    c = Cache(128, 4, [70] * 40, 64)
    for _ in range(67):
        c.append([1] * 40, uniform=True)
    c.check()
    c.close()


@pytest.mark.parametrize("sequences", [1, 31, 32, 33, 64, 65, 1024, 1025, 2100])
def test_rows_find_their_sequence(sequences):
    """Sequences at the borders of what a warp looks through at once, some of them empty (the first and the last, and runs of more than a warp)."""
    ns = [0 if sequences > 1 and (i in (0, sequences - 1) or i % 3 == 1 or 40 <= i < 110) else 1 + 31 * (i % 11 == 5) + 40 * (i % 13 == 2)
          for i in range(sequences)]
    c = Cache(8, 1, [1 + 2 * n for n in ns])
    for n in (ns, [min(1, x) for x in ns], ns):
        c.append(n)
    c.check()
    c.close()


@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_exponents_at_their_ends(dtype):
    """Borders of the exponent (127 2^e and the next number above), nothing but zeros, the smallest and largest magnitudes."""
    c = Cache(16, 2, [32 * 12], 32)
    up = lambda x: np.nextafter(np.float32(x), np.float32(np.inf)) if dtype == "f32" else np.nextafter(np.float16(x), np.float16(np.inf))
    big = 65504.0 if dtype == "f16" else 3e38
    for top in (0.0, 2.0 ** -24, 127 * 2.0 ** -20, up(127 * 2.0 ** -20), 127.0, up(127.0), 126.5, 128.0, 127 * 2.0 ** 8, up(127 * 2.0 ** 8), 65024.0, big):
        def make(n):
            x = np.zeros((n, 2, 16))
            x[:, 0, 3] = top
            x[n // 2, 1, 5] = -float(top) / 3
            x[:, :, 7] = float(top) / 254        # a tie: half a step where the step is top / 127
            return x
        c.append([32], dtype, make=make)
    c.check()
    c.close()


def test_layers_are_apart():
    a = Cache(64, 2, [50], 32, layers=3, layer=1)
    a.append([40])
    held = a.held
    for layer in (0, 2):
        a.layer, a.held = layer, [[np.zeros_like(x) for x in side] for side in held]
        a.check()
    a.layer, a.held = 1, held
    a.check()
    a.close()


def test_a_page_begun_anew_forgets():
    """A page that another sequence has used: its first block's old exponent and codes count no more."""
    c = Cache(64, 2, [32], 32)
    c.append([32], make=lambda n: 30 * c.values(n))
    c.len, c.exps = [0], [[{}], [{}]]
    c.append([3], make=lambda n: 0.01 * c.values(n))
    c.check()
    c.append([1], make=lambda n: 0.01 * c.values(n))
    c.check()
    c.close()


# ---- attention -------------------------------------------------------------------------------------------------------
def attend(q, k, v, scale, place, causal, window, sinks):
    """q [n][hq][D], k and v [len][hk][D] in 64 bits -> (out, how far an element may be from it).  u = 2^-24.  A product of D terms on the tensor
    cores is within 2 D u of the sum of their magnitudes, and what becomes of it (scale, difference, power) within 8 u of the exponent's magnitude:
    that moves a weight by so much of itself.  A weight is rounded to a half: 2^-11 of it, or 2^-25 of the largest where it is that small.  Sums and joins
    of n terms: 2 sqrt(n) + 64 roundings."""
    u = 2.0 ** -24
    n, hq, D = q.shape
    g = hq // max(1, k.shape[1])
    out, err = np.zeros((n, hq, D)), np.zeros((n, hq, D))
    t = np.arange(len(k))
    seen = np.ones((n, len(k)), bool)
    if causal:
        p = place + np.arange(n)[:, None]
        seen = t <= p
        if window:
            seen &= (t > p - window) | (t < sinks)
    for h in range(hq):
        kh, vh = k[:, h // g], v[:, h // g]
        if len(k) == 0:
            continue
        s = np.where(seen, q[:, h] @ kh.T * scale, -np.inf)
        mag = np.abs(q[:, h]) @ np.abs(kh).T * abs(scale)
        top = s.max(1, keepdims=True)
        w = np.exp(s - top)
        off = (2 * D + 16) * u * np.where(seen, mag, 0).max(1, keepdims=True) + 16 * u
        total = w.sum(1, keepdims=True)
        out[:, h] = w @ vh / total
        near = w @ np.abs(vh) / total
        small = seen.sum(1, keepdims=True) * 2.0 ** -25 * np.abs(vh).max() / total
        err[:, h] = (2.0 ** -11 + 2 * off + (2 * np.sqrt(len(k)) + 64) * u) * near + small
    return out, err + (np.abs(out) + err) * 2.0 ** -11 + 2.0 ** -25


def run_attention(c, ns, lens, hq, causal=True, window=0, sinks=0, uniform=False, behind=0, scale=None, apart=False, call=None):
    """Queries inside a projection's rows, or heads apart; the output's rows behind the last sequence stay."""
    import torch
    rows = sum(ns) + behind
    q = (c.rng.standard_normal((rows, hq, c.D)) * 1.5).astype(np.float16)
    scale = c.D ** -0.5 if scale is None else scale
    if apart:
        qd = torch.from_numpy(np.ascontiguousarray(q.transpose(1, 0, 2))).cuda()
        st = (qd.stride(1), qd.stride(0))
        out = torch.full((hq, rows, c.D + 8), 7.0, dtype=torch.float16, device="cuda")
        so = (out.stride(1), out.stride(0))
        view = lambda: out[:, :, : c.D].transpose(0, 1)
    else:
        qd = torch.zeros(rows, hq + 3, c.D, dtype=torch.float16, device="cuda")
        qd[:, :hq] = torch.from_numpy(q).cuda()
        st = qd.stride()[:2]
        out = torch.full((rows, hq, c.D), 7.0, dtype=torch.float16, device="cuda")
        so = out.stride()[:2]
        view = lambda: out
    b = c.batch(ns, lens, uniform, behind)
    a = B.lq_attn(qd.data_ptr(), st, out.data_ptr(), so, hq, scale, causal, window, sinks)
    B.lq_cache_attention(c.h, c.layer, b, a, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    got = view().float().cpu().numpy().astype(np.float64)
    if apart:
        assert (out[:, :, c.D:] == 7).all()
    at = 0
    for s, (n, t) in enumerate(zip(ns, lens)):
        want, err = attend(q[at:at + n].astype(np.float64), c.held[0][s][:t], c.held[1][s][:t], scale, t - n, causal, window, sinks)
        far = np.abs(got[at:at + n] - want) / err
        assert n == 0 or far.max() <= 1, (s, float(far.max()), np.unravel_index(far.argmax(), far.shape))
        at += n
    assert (got[at:] == 7).all()
    return got


def filled(D, heads, lens, page=32, seed=0):
    c = Cache(D, heads, lens, page, seed=seed)
    c.append(list(lens))
    return c


@pytest.mark.parametrize("D,hq,hk", [(8, 1, 1), (16, 2, 2), (64, 8, 2), (72, 4, 4), (80, 10, 2), (96, 6, 3), (112, 7, 1), (128, 32, 8), (128, 40, 2),
                                     (160, 4, 2), (192, 3, 1), (256, 16, 4)])
def test_single_tokens(D, hq, hk):
    lens = [1, 2, 31, 32, 33, 64, 100, 257, 600]
    c = filled(D, hk, lens, 64)
    run_attention(c, [1] * len(lens), lens, hq, uniform=True)
    run_attention(c, [1] * len(lens), lens, hq, apart=True)
    c.close()


@pytest.mark.parametrize("length", [1, 255, 4096, 9001])
def test_one_sequence_over_the_whole_grid(length):
    """Its records are many blocks' of the grid, which join their parts; equal calls give equal bits."""
    c = filled(128, 2, [length], 128)
    a = run_attention(c, [1], [length], 8)
    c.rng = np.random.default_rng(5)
    a = run_attention(c, [1], [length], 8)
    c.rng = np.random.default_rng(5)
    assert np.array_equal(a, run_attention(c, [1], [length], 8))
    c.close()


@pytest.mark.parametrize("D,hq,hk,page", [(64, 4, 1, 32), (72, 6, 6, 32), (128, 8, 2, 64), (112, 14, 2, 96), (192, 4, 2, 32), (256, 4, 4, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (40, 0), (100, 4), (64, 70), (5000, 3)])
def test_prompts_and_masks(D, hq, hk, page, window, sinks):
    """Several new tokens, none, one; sequences that begin with them and that have more; rows behind the last sequence."""
    lens, ns = [1, 40, 300, 0, 129, 513, 200], [1, 40, 3, 0, 129, 200, 65]
    c = filled(D, hk, lens, page)
    run_attention(c, ns, lens, hq, True, window, sinks, behind=3)
    c.close()


@pytest.mark.parametrize("D,hq,hk", [(72, 4, 4), (128, 8, 2), (256, 2, 1)])
def test_every_token_sees_every_other(D, hq, hk):
    """Also rows of other sequences' (as many as they like, of a length of none, too)."""
    lens, ns = [256, 1, 33, 0, 700, 64], [256, 5, 200, 3, 31, 0]
    c = filled(D, hk, lens)
    run_attention(c, ns, lens, hq, False, behind=1)
    run_attention(c, [64] * 6, lens, hq, False, uniform=True, apart=True)
    c.close()


@pytest.mark.parametrize("D,hq,hk,window,sinks", [(128, 8, 2, 0, 0), (72, 2, 2, 0, 0), (64, 8, 1, 1500, 40), (96, 3, 1, 700, 0), (112, 6, 2, 0, 0)])
def test_few_tiles_of_rows_over_a_long_cache(D, hq, hk, window, sinks):
    """Tiles of rows that many thread blocks share; one sequence of one length, ragged ones, some with rows of the other form, all and causal."""
    lens = [4500, 90, 2500]
    c = filled(D, hk, lens, 64)
    for ns in ([70, 0, 0], [100, 90, 300], [3, 1, 200]):
        run_attention(c, ns, lens, hq, True, window, sinks, behind=2)
        if not window:
            run_attention(c, ns, lens, hq, False)
    run_attention(c, [90, 90, 90], lens, hq, True, window, sinks, uniform=True)
    c.close()


@pytest.mark.parametrize("sequences", [300, 1000])
def test_many_sequences(sequences):
    lens = [1 + (37 * i) % 90 for i in range(sequences)]
    ns = [(i % 7 != 0) * (1 + (i % 5 == 0) * min(lens[i] - 1, 4)) for i in range(sequences)]
    c = filled(64, 1, lens, 32)
    run_attention(c, ns, lens, 2)
    c.close()


@pytest.mark.parametrize("D,hq,hk", [(128, 4, 1), (80, 2, 2), (64, 8, 1)])
def test_equal_calls_give_equal_bits(D, hq, hk):
    """Prompts, again and again: operands are whole when they are read, whatever the order in which copies and warps come."""
    import torch
    c = filled(D, hk, [513, 300, 100], 64)
    ns = [200, 300, 1]
    q = torch.randn(sum(ns), hq, D, dtype=torch.float16, device="cuda")
    out = torch.empty(2, sum(ns), hq, D, dtype=torch.float16, device="cuda")
    b = c.batch(ns, c.len)
    for i in range(300):
        a = B.lq_attn(q.data_ptr(), q.stride()[:2], out[min(i, 1)].data_ptr(), out.stride()[1:3], hq, 0.1)
        B.lq_cache_attention(c.h, 0, b, a, torch.cuda.current_stream().cuda_stream)
        assert i == 0 or torch.equal(out[0], out[1]), i
    c.close()


def test_heavy_rows_and_large_products():
    """One token takes all the weight (a difference of exponents beyond fp32's range); values of very different size."""
    c = Cache(64, 1, [200], 32)
    def make(n):
        x = c.values(n)
        x[50] *= 40
        return x
    c.append([200], make=make)
    run_attention(c, [3], [200], 2, scale=4.0)
    run_attention(c, [3], [200], 2, scale=0.0)
    run_attention(c, [3], [200], 2, scale=-0.5)
    c.close()


def test_masked_places_may_hold_anything():
    """What lies behind a sequence's tokens in its last block, or is left of another sequence there, reaches no output."""
    c = Cache(64, 2, [64], 32)
    c.append([64], make=lambda n: np.full((n, 2, 64), 65504.0))
    c.len, c.exps = [0], [[{}], [{}]]
    c.append([33])
    run_attention(c, [5], [33], 4)
    run_attention(c, [5], [33], 4, causal=False)
    c.close()


def test_arrays_that_do_not_fit_are_left_out():
    """Lengths beyond the pages or below the rows, pages that are none: the others are right, and the status word says so."""
    import torch
    lens = [40, 50, 60, 70]
    c = filled(64, 2, lens, 32)
    assert B.lq_get_device_status(0) == (0, 0)
    for bad in ("long", "negative", "short", "page", "page -1"):
        ns, tell = [2, 2, 2, 2], list(lens)
        pages = c.pages.copy()
        if bad == "long":
            tell[1] = c.stride * 32 + 1
        elif bad == "negative":
            tell[1] = -5
        elif bad == "short":
            tell[1] = 1
        else:
            pages[1, 0] = c.pages.max() + 1000 if bad == "page" else -1
        keep = c.pages_d
        c.pages_d = torch.from_numpy(pages).cuda()
        b = c.batch(ns, tell)
        x = torch.randn(8, 4, 64, dtype=torch.float16, device="cuda")
        out = torch.full_like(x, 7.0)
        st = torch.cuda.current_stream().cuda_stream
        B.lq_cache_attention(c.h, 0, b, B.lq_attn(x.data_ptr(), (256, 64), out.data_ptr(), (256, 64), 4, 0.1), st)
        torch.cuda.synchronize()
        assert B.lq_get_device_status(0)[0] == 1, bad
        if not bad.startswith("page"):
            assert (out[2:4] == 7).all()
        xs = x.double().cpu().numpy()
        for s in (0, 2, 3):
            want, err = attend(xs[2 * s:2 * s + 2], c.held[0][s][:lens[s]], c.held[1][s][:lens[s]], 0.1, lens[s] - 2, True, 0, 0)
            assert (np.abs(out[2 * s:2 * s + 2].double().cpu().numpy() - want) <= err).all(), (bad, s)
        # the same to write and to read: only what fits
        B.lq_kvcache_append(c.h, 0, b, B.lq_kvrows(x.data_ptr(), (0, 256, 64), x.data_ptr(), (0, 256, 64)), B.OUT_F16, st)
        torch.cuda.synchronize()
        assert B.lq_get_device_status(0)[0] == (0 if bad.startswith("page") else 1), bad      # (the page that is none is not written)
        read = torch.zeros(2, 4, 70, 2, 64, device="cuda")
        rst = (read.stride(1), read.stride(2), read.stride(3))
        B.lq_kvcache_read(c.h, 0, b, None, 70, B.lq_kvrows(read[0].data_ptr(), rst, read[1].data_ptr(), rst), B.OUT_F32, st)
        torch.cuda.synchronize()
        assert B.lq_get_device_status(0)[0] == (0 if bad == "short" else 1), bad
        c.pages_d = keep
        for s in range(4):                                 # back to what the oracle holds
            c.len[s] = lens[s] - 2
        c = _rewritten(c, lens)
    c.close()


def _rewritten(c, lens):
    c.len, c.exps = [0] * c.B, [[{} for _ in lens] for _ in "kv"]
    c.append(list(lens))
    return c


def test_a_captured_step_goes_by_what_the_arrays_hold():
    """Append and attention in one graph; lengths and rows change between replays."""
    import torch
    lens = [5, 90, 31]
    c = Cache(128, 2, [40, 120, 70], 32)
    c.append(lens)
    x = torch.zeros(3, 12, 128, dtype=torch.float16, device="cuda")
    out = torch.zeros(3, 8, 128, dtype=torch.float16, device="cuda")
    ld = torch.tensor(lens, dtype=torch.int32, device="cuda")
    b = B.lq_kvbatch(3, 3, ld.data_ptr(), c.pages_d.data_ptr(), c.stride)
    a = B.lq_attn(x.data_ptr(), x.stride()[:2], out.data_ptr(), out.stride()[:2], 8, 0.1)
    rows = B.lq_kvrows(x[:, 8:].data_ptr(), (0, *x.stride()[:2]), x[:, 10:].data_ptr(), (0, *x.stride()[:2]))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        ld.add_(1)
        B.lq_kvcache_append(c.h, 0, b, rows, B.OUT_F16, side.cuda_stream)
        B.lq_cache_attention(c.h, 0, b, a, side.cuda_stream)
    for step in range(30):
        new = (c.rng.standard_normal((3, 12, 128)) * np.exp(c.rng.standard_normal((3, 1, 1)))).astype(np.float16)
        x.copy_(torch.from_numpy(new))
        graph.replay()
        torch.cuda.synchronize()
        lens = [n + 1 for n in lens]
        for s in range(3):
            for side_i, cols in ((0, slice(8, 10)), (1, slice(10, 12))):
                write(c.held[side_i][s], c.exps[side_i][s], new[s:s + 1, cols].astype(np.float64), lens[s] - 1)
            want, err = attend(new[s:s + 1, :8].astype(np.float64), c.held[0][s][:lens[s]], c.held[1][s][:lens[s]], 0.1, lens[s] - 1, True, 0, 0)
            assert (np.abs(out[s:s + 1].double().cpu().numpy() - want) <= err).all(), (step, s)
    del graph
    c.len = lens
    c.check()
    c.close()


def test_offsets_beyond_32_bits():
    """Records behind 2^32 bytes, rows of queries and outputs behind 2^31 elements; prompts, single tokens, writing and reading."""
    import torch
    D, H, n_pages = 128, 4, 48000
    h = B.lq_kvcache_create(2, n_pages, 64, H, D)           # 3.2 GB a layer
    c = Cache(D, H, [300, 200], 64)
    B.lq_kvcache_free(c.h)
    c.h, c.layer = h, 1
    c.pages = np.where(c.pages >= 0, n_pages - 1 - c.pages, -1).astype(np.int32)
    c.pages_d = torch.from_numpy(c.pages).cuda()
    c.append([300, 200])
    c.check()
    far = 1 << 24                                          # times 190 rows passes 2^31 elements
    buf = torch.empty(2, 191 * far, dtype=torch.float16, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    for ns in ([150, 40], [1, 1]):
        rows = sum(ns)
        q = c.rng.standard_normal((rows, 4, D)).astype(np.float16)
        qf, of = (torch.as_strided(x, (rows, 4, D), (far, D, 1), x.storage_offset()) for x in buf)
        qf.copy_(torch.from_numpy(q).cuda())
        b = c.batch(ns, c.len)
        B.lq_cache_attention(c.h, 1, b, B.lq_attn(buf[0].data_ptr(), (far, D), buf[1].data_ptr(), (far, D), 4, 0.1), st)
        got, at = of.double().cpu().numpy(), 0
        for s, n in enumerate(ns):
            want, err = attend(q[at:at + n].astype(np.float64), c.held[0][s][:c.len[s]], c.held[1][s][:c.len[s]], 0.1, c.len[s] - n, True, 0, 0)
            assert (np.abs(got[at:at + n] - want) <= err).all(), s
            at += n
    c.close()


def test_refusals():
    import torch
    code = lambda f, *a: _code(f, *a)
    for bad, want in (((0, 1, 32, 1, 64), 1), ((1, 0, 32, 1, 64), 1), ((1, 1, 0, 1, 64), 1), ((1, 1, 32, 0, 64), 1), ((1, 1, 32, 1, 0), 1), ((1, 1, 33, 1, 64), 2),
                      ((1, 1, 32, 1, 60), 2), ((1, 1, 32, 1, 264), 2), ((1, 1, 32, 5000, 64), 2), ((1, 2 ** 30, 65536, 64, 256), 3), ((1, 1, 32, 1, 64, 99), 4)):
        assert code(B.lq_kvcache_create, *bad) == want, bad
    c = Cache(64, 2, [100], 32)
    x = torch.zeros(8, 8, 64, dtype=torch.float16, device="cuda")
    out = torch.zeros(8, 4, 64, dtype=torch.float16, device="cuda")
    ints = torch.zeros(16, dtype=torch.int32, device="cuda")
    batch = lambda s=1, rows=1, length=ints.data_ptr(), pages=ints.data_ptr(), stride=4, start=None: B.lq_kvbatch(s, rows, length, pages, stride, start)
    rows = lambda k=x.data_ptr(), v=x.data_ptr(), st=(0, 512, 64): B.lq_kvrows(k, st, v, st)
    attn = lambda q=x.data_ptr(), sq=(512, 64), o=out.data_ptr(), so=(256, 64), hq=4, scale=0.1, **k: B.lq_attn(q, sq, o, so, hq, scale, **k)
    nan, big = float("nan"), 1 << 40
    for b, want in ((batch(0), 1), (batch(1, -1), 1), (batch(3, 4), 1), (batch(length=0), 1), (batch(pages=0), 1), (batch(stride=0), 1), (batch(70000, 70000), 2),
                    (batch(length=ints.data_ptr() + 2), 1), (batch(start=ints.data_ptr() + 1), 1)):
        assert code(B.lq_kvcache_append, c.h, 0, b, rows()) == want
        assert code(B.lq_kvcache_read, c.h, 0, b, None, 1, rows()) == want
        assert code(B.lq_cache_attention, c.h, 0, b, attn()) == want
    for layer in (-1, 1):
        assert code(B.lq_cache_attention, c.h, layer, batch(), attn()) == 1 and code(B.lq_kvcache_append, c.h, layer, batch(), rows()) == 1
    for r, want in ((rows(k=0), 1), (rows(v=0), 1), (rows(k=x.data_ptr() + 8), 1), (rows(st=(0, 516, 64)), 1), (rows(st=(0, 512, 4)), 1), (rows(st=(0, big, 64)), 2)):
        assert code(B.lq_kvcache_append, c.h, 0, batch(), r) == want
    assert code(B.lq_kvcache_append, c.h, 0, batch(), rows(), 2) == 1
    assert code(B.lq_kvcache_read, c.h, 0, batch(), None, 0, rows()) == 1 and code(B.lq_kvcache_read, c.h, 0, batch(), None, 4, rows(k=0, v=0)) == 1
    assert code(B.lq_kvcache_read, c.h, 0, batch(), None, 4, rows()) == 1                           # both on one place
    assert code(B.lq_kvcache_read, c.h, 0, batch(), None, 4, rows(v=0, st=(0, 64, 64))) == 1        # rows and heads on one place
    for a, want in ((attn(q=0), 1), (attn(o=0), 1), (attn(hq=3), 1), (attn(hq=0), 1), (attn(hq=8192), 2), (attn(scale=nan), 1), (attn(scale=float("inf")), 1),
                    (attn(window=-1), 1), (attn(sinks=-1, window=3), 1), (attn(sinks=1), 1), (attn(causal=False, window=3), 1), (attn(q=x.data_ptr() + 2), 1),
                    (attn(sq=(508, 64)), 1), (attn(so=(256, 60)), 1), (attn(so=(big, 64)), 2), (attn(o=x.data_ptr(), so=(512, 64)), 1), (attn(so=(256, 8)), 1)):
        assert code(B.lq_cache_attention, c.h, 0, batch(), a) == want
    assert code(B.lq_cache_attention, c.h, 0, batch(2, 4), attn(so=(128, 64))) == 1
    B.lq_cache_attention(c.h, 0, batch(rows=0), attn())                                            # nothing to do
    B.lq_kvcache_append(c.h, 0, batch(rows=0), rows())
    c.close()


def _code(f, *a):
    with pytest.raises(B.LqError) as e:
        f(*a)
    return e.value.code
