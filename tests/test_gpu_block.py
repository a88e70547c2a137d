"""What an attention block does around its quantized projections, in one run: norm, queries, keys and values, cache, attention, output projection, sum and
norm; a prompt, then single tokens in a captured graph."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

from .test_gpu_kvcache import attend, write

pytestmark = pytest.mark.gpu

HIDDEN, HQ, HK, D, EPS = 512, 8, 2, 64, 1e-6


def make_layer(K, N, seed):
    """A SINT4 layer of random codes and no branch."""
    rng = np.random.default_rng(seed)
    W = (rng.standard_normal((K, N)) / np.sqrt(K)).astype(np.float16)
    cfg = B.lq_config_default(K, N, 0, "none")
    cfg.steps = 0
    h, _ = B.lq_calibrate(cfg, W)
    B.lq_layer_to_device(h, 0)
    return h


class Block:
    def __init__(self, lens, new, layer=1):
        import torch
        self.B, self.n, self.layer = len(lens), new, layer
        self.qkv = make_layer(HIDDEN, (HQ + 2 * HK) * D, 1)
        self.out = make_layer(HQ * D, HIDDEN, 2)
        self.rows = self.B * new
        self.acts = [B.lq_act_create(h, self.rows, 0) for h in (self.qkv, self.out)]
        self.x = torch.zeros(self.rows, HIDDEN, device="cuda")
        self.h, self.y, self.h1 = (torch.zeros(self.rows, HIDDEN, dtype=torch.float16, device="cuda") for _ in range(3))
        self.z = torch.zeros(self.rows, (HQ + 2 * HK) * D, dtype=torch.float16, device="cuda")
        self.a = torch.zeros(self.rows, HQ * D, dtype=torch.float16, device="cuda")
        rng = np.random.default_rng(3)
        self.mod = (0.3 * rng.standard_normal((self.B, 3, HIDDEN))).astype(np.float32)
        self.w = (1 + 0.2 * rng.standard_normal(HIDDEN)).astype(np.float32)
        self.mod_d, self.w_d = torch.from_numpy(self.mod).cuda(), torch.from_numpy(self.w).cuda()
        self.rope = B.lq_rope_create(B.lq_rope_config_default([D], halves=True))
        self.pos = torch.zeros(self.rows, 1, dtype=torch.int32, device="cuda")
        self.length = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def run(self, cache, pages, stream):
        shift, scale, gate = (self.mod_d[:, i].data_ptr() for i in range(3))
        norm = dict(sequences=self.B, norm=B.NORM_RMS, weight_ptr=self.w_d.data_ptr(), shift_ptr=shift, scale_ptr=scale, mod_seq=3 * HIDDEN, eps=EPS,
                    x_dtype=B.OUT_F32, mod_dtype=B.OUT_F32)
        B.lq_residual_norm(B.lq_residual(self.rows, HIDDEN, self.x.data_ptr(), None, self.h.data_ptr(), **norm), stream)
        q = B.lq_qkv(D, HQ, HK, self.B, B.NORM_RMS, EPS, self.rope, self.pos.data_ptr())
        B.lq_qkv_forward(self.qkv, self.acts[0], self.h.data_ptr(), self.rows, None, None, q, self.z.data_ptr(), B.OUT_F16, stream)
        b = B.lq_kvbatch(self.B, self.rows, self.length.data_ptr(), pages.data_ptr(), pages.shape[1])
        row = self.z.shape[1]
        B.lq_kvcache_append(cache, self.layer, b, B.lq_kvrows(self.z[:, HQ * D:].data_ptr(), (0, row, D), self.z[:, (HQ + HK) * D:].data_ptr(), (0, row, D)),
                            B.OUT_F16, stream)
        B.lq_cache_attention(cache, self.layer, b, B.lq_attn(self.z.data_ptr(), (row, D), self.a.data_ptr(), (HQ * D, D), HQ, D ** -0.5), stream)
        B.lq_quantize_act(self.out, self.a.data_ptr(), self.rows, self.acts[1], stream)
        B.lq_linear_forward(self.out, self.acts[1], self.y.data_ptr(), B.OUT_F16, stream)
        B.lq_residual_norm(B.lq_residual(self.rows, HIDDEN, self.x.data_ptr(), self.x.data_ptr(), self.h1.data_ptr(), y_ptr=self.y.data_ptr(), gate_ptr=gate,
                                         **norm), stream)

    def free(self):
        for a in self.acts:
            B.lq_act_free(a)
        B.lq_layer_free(self.qkv)
        B.lq_layer_free(self.out)
        B.lq_rope_free(self.rope)


def normed(x, w, shift, scale):
    return x / np.sqrt(np.square(x).mean(-1, keepdims=True) + EPS) * w * (1 + scale) + shift


def check(blk, x0, lens, held, exps, before):
    """Step by step from what the step before has put out, so that no rounding is passed on: each within its own bound."""
    n, Bn = blk.n, blk.B
    get = lambda t: t.double().cpu().numpy()
    z, a, x1, y, h0, h1 = (get(t) for t in (blk.z, blk.a, blk.x, blk.y, blk.h, blk.h1))
    per = lambda i: np.repeat(blk.mod[:, i].astype(np.float64), n, 0)
    want = normed(x0, blk.w, per(0), per(1))
    # a sum of 512 terms in a tree and some ten operations of fp32, rounded to a half
    assert (np.abs(h0 - want) <= (64 * 2.0 ** -24 + 2.0 ** -11) * (np.abs(want) + np.abs(per(0)) + np.abs(want - per(0))) + 2.0 ** -25).all()
    for s in range(Bn):
        rows = slice(s * n, s * n + n)
        zs = z[rows].reshape(n, HQ + 2 * HK, D)
        for side in range(2):
            write(held[side][s], exps[side][s], zs[:, HQ + side * HK:HQ + (side + 1) * HK], before[s])
        want, err = attend(zs[:, :HQ], held[0][s][:lens[s]], held[1][s][:lens[s]], D ** -0.5, lens[s] - n, True, 0, 0)
        assert (np.abs(a[rows].reshape(n, HQ, D) - want) <= err).all(), s
    # the sum: a product, an addition, in fp32; the projection's output is some part of it
    assert (np.abs(x1 - (x0 + per(2) * y)) <= 2 * 2.0 ** -24 * (np.abs(x1) + np.abs(per(2) * y))).all() and np.abs(y).max() > 0
    want = normed(x1, blk.w, per(0), per(1))               # (x1 is held in fp32: the norm's input but for its rounding, which the 64 roundings cover)
    assert (np.abs(h1 - want) <= (64 * 2.0 ** -24 + 2.0 ** -11) * (np.abs(want) + np.abs(per(0)) + np.abs(want - per(0))) + 2.0 ** -25).all()


def test_a_block_over_a_prompt_and_single_tokens():
    import torch
    st = torch.cuda.current_stream().cuda_stream
    prompt, steps, Bn = 70, 40, 3
    cache = B.lq_kvcache_create(2, 4 * Bn, 32, HK, D)
    order = np.random.default_rng(9).permutation(4 * Bn).astype(np.int32).reshape(Bn, 4)
    pages = torch.from_numpy(order).cuda()
    held = [[np.zeros((128, HK, D)) for _ in range(Bn)] for _ in "kv"]
    exps = [[{} for _ in range(Bn)] for _ in "kv"]
    rng = np.random.default_rng(4)

    first = Block([prompt] * Bn, prompt)
    x = rng.standard_normal((Bn * prompt, HIDDEN)).astype(np.float32)
    first.x.copy_(torch.from_numpy(x))
    first.pos.copy_(torch.arange(prompt, dtype=torch.int32).repeat(Bn)[:, None])
    first.run(cache, pages, st)
    torch.cuda.synchronize()
    check(first, x.astype(np.float64), [prompt] * Bn, held, exps, [0] * Bn)
    first.free()

    one = Block([prompt] * Bn, 1)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        one.pos.copy_(one.length[:, None])
        one.length.add_(1)
        one.run(cache, pages, side.cuda_stream)
    for i in range(steps):
        x = rng.standard_normal((Bn, HIDDEN)).astype(np.float32)
        one.x.copy_(torch.from_numpy(x))
        graph.replay()
        torch.cuda.synchronize()
        check(one, x.astype(np.float64), [prompt + i + 1] * Bn, held, exps, [prompt + i] * Bn)
    del graph
    one.free()
    assert B.lq_get_device_status(0) == (0, 0)
    B.lq_kvcache_free(cache)


def test_two_caches_on_two_streams():
    """Calls of distinct caches side by side: each as by itself, to the bit."""
    import torch
    rng = np.random.default_rng(5)
    caches, want, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for i, (lens, n) in enumerate((([900, 40], 1), ([500, 333], 100))):
        H, pages = 2, torch.arange(2 * 16, dtype=torch.int32, device="cuda").view(2, 16)
        c = B.lq_kvcache_create(1, 32, 64, H, D)
        kv = torch.from_numpy(rng.standard_normal((2, 1000, 2 * H, D)).astype(np.float16)).cuda()
        length, q = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.randn(2 * n, HQ, D, dtype=torch.float16, device="cuda")
        start = torch.tensor([0, lens[0], sum(lens)], dtype=torch.int32, device="cuda")
        kv = kv.view(2000, 2 * H, D)
        b0 = B.lq_kvbatch(2, sum(lens), length.data_ptr(), pages.data_ptr(), 16, start.data_ptr())
        B.lq_kvcache_append(c, 0, b0, B.lq_kvrows(kv.data_ptr(), (0, 2 * H * D, D), kv[:, H:].data_ptr(), (0, 2 * H * D, D)))
        out = torch.zeros(50, 2 * n, HQ, D, dtype=torch.float16, device="cuda")
        call = lambda o, s, c=c, q=q, n=n, length=length, pages=pages: B.lq_cache_attention(
            c, 0, B.lq_kvbatch(2, 2 * n, length.data_ptr(), pages.data_ptr(), 16), B.lq_attn(q.data_ptr(), (HQ * D, D), o.data_ptr(), (HQ * D, D), HQ, 0.125), s)
        torch.cuda.synchronize()
        call(out[0], streams[0].cuda_stream)
        torch.cuda.synchronize()
        want.append(out[0].clone())
        caches.append((c, call, out, (kv, start)))
    for i in range(50):
        for (c, call, out, _), s in zip(caches, streams):
            call(out[i], s.cuda_stream)
    torch.cuda.synchronize()
    for (c, call, out, _), w in zip(caches, want):
        assert (out == w).all()
        B.lq_kvcache_free(c)
