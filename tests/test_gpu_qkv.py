"""The projection of an attention block as it is served: quantized linear, the requests' adapters, norms and rotation, in one call and one by one."""
import numpy as np
import pytest

from oracle import lq_oracle as O
from paper_2604_18117_b200 import binding as B
from tests.helpers import import_oracle_layer

pytestmark = pytest.mark.gpu


def _layer(rng, K, N, r):
    layer = {"branch": "w8a8", "rank": r, "K": K, "N": N, "bias": (rng.standard_normal(N) * 0.05).astype(np.float16)}
    layer["Wq"], layer["sw"] = O.q_weight_main(rng.standard_normal((K, N)) * 0.02)
    layer["L1q"], layer["sL1"] = O.q_factor(rng.standard_normal((K, r)) * 0.05, 8)
    layer["L2q"], layer["sL2"] = O.q_factor(rng.standard_normal((r, N)) * 0.05, 8)
    return layer


class Block:
    """heads of 72 on 288 features, two adapters, two position axes; everything on the GPU"""

    def __init__(self, M, sequences, f32, hq=4, hk=4, D=72, seed=0):
        import torch
        rng = np.random.default_rng(seed + M)
        self.K, self.M, self.seqs, self.hq, self.hk, self.D, self.f32 = hq * D, M, sequences, hq, hk, D, f32
        self.N = (hq + 2 * hk) * D
        self.layer = _layer(rng, self.K, self.N, 16)
        self.h, _ = import_oracle_layer(self.layer)
        B.lq_layer_to_device(self.h, 0)
        self.act = B.lq_act_create(self.h, M, 0)
        self.set, self.map = B.lq_adapters_create(self.K, self.N, 16, 2, 0), B.lq_rowmap_create(M, 2, 0)
        self.A = (rng.standard_normal((2, self.K, 16)) * 0.02).astype(np.float16)
        self.Bf = (rng.standard_normal((2, 16, self.N)) * 0.2).astype(np.float16)
        self.kept = [torch.from_numpy(x).cuda() for x in (self.A, self.Bf)]
        st = torch.cuda.current_stream().cuda_stream
        for i in range(2):
            B.lq_adapters_set(self.set, i, 16, self.kept[0][i].data_ptr(), self.kept[1][i].data_ptr(), 0.5 + i, st)
        self.ids = rng.integers(-1, 2, M).astype(np.int32)
        self.X = rng.standard_normal((M, self.K)).astype(np.float16)
        self.pos = rng.integers(0, 5000, (M, 2)).astype(np.int32)
        self.w = (1 + 0.3 * rng.standard_normal((2, D))).astype(np.float32)
        self.x, self.i, self.p, self.wd = (torch.from_numpy(v).cuda() for v in (self.X, self.ids, self.pos, self.w))
        self.rope = B.lq_rope_create(B.lq_rope_config_default([36, 36]), 0)
        self.y = [torch.full((M, self.N), float("nan"), dtype=torch.float32 if f32 else torch.float16, device="cuda") for _ in range(2)]
        self.code = B.OUT_F32 if f32 else B.OUT_F16
        self.qkv = B.lq_qkv(D, hq, hk, sequences, B.NORM_RMS, 1e-6, self.rope, self.p.data_ptr(), self.wd[0].data_ptr(), self.wd[1].data_ptr())

    def one_call(self, y, st, adapters=True):
        B.lq_rowmap_set(self.map, self.i.data_ptr(), self.M, st)
        B.lq_qkv_forward(self.h, self.act, self.x.data_ptr(), self.M, self.set if adapters else None, self.map if adapters else None, self.qkv, y.data_ptr(), self.code, st)

    def one_by_one(self, y, st, adapters=True):
        B.lq_quantize_act(self.h, self.x.data_ptr(), self.M, self.act, st)
        B.lq_linear_forward(self.h, self.act, y.data_ptr(), self.code, st)
        if adapters:
            B.lq_rowmap_set(self.map, self.i.data_ptr(), self.M, st)
            B.lq_adapters_forward(self.set, self.map, self.x.data_ptr(), y.data_ptr(), y.data_ptr(), self.code, st)
        S, esz = self.M // self.seqs, y.element_size()
        strides = (S * self.N, self.N, self.D)
        q = B.lq_heads(y.data_ptr(), strides, y.data_ptr(), strides, self.hq, self.wd[0].data_ptr())
        at = y.data_ptr() + self.hq * self.D * esz
        k = B.lq_heads(at, strides, at, strides, self.hk, self.wd[1].data_ptr())
        B.lq_qk_norm_rope(q, k, self.D, self.seqs, S, B.NORM_RMS, 1e-6, self.rope, self.p.data_ptr(), self.code, self.code, st)

    def formula(self):
        """In 64 bits, from the oracle's forward on."""
        Y = O.forward(self.X, self.layer)["Y"].astype(np.float64)
        for a in range(2):
            r = self.ids == a
            Y[r] += (0.5 + a) * (self.X[r].astype(np.float64) @ self.A[a].astype(np.float64) @ self.Bf[a].astype(np.float64))
        heads = Y.reshape(self.M, self.hq + 2 * self.hk, self.D)
        freq = 10000.0 ** (-2 * np.arange(18) / 36)
        t = np.concatenate([self.pos[:, :1] * freq, self.pos[:, 1:] * freq], 1)[:, None]
        for lo, hi, w in ((0, self.hq, self.w[0]), (self.hq, self.hq + self.hk, self.w[1])):
            z = heads[:, lo:hi]
            z = z / np.sqrt(np.square(z).mean(-1, keepdims=True) + 1e-6) * w
            u, v = z[..., 0::2].copy(), z[..., 1::2].copy()
            z[..., 0::2], z[..., 1::2] = u * np.cos(t) - v * np.sin(t), v * np.cos(t) + u * np.sin(t)
            heads[:, lo:hi] = z
        return heads.reshape(self.M, self.N)

    def free(self):
        for f, h in ((B.lq_act_free, self.act), (B.lq_layer_free, self.h), (B.lq_adapters_free, self.set), (B.lq_rowmap_free, self.map), (B.lq_rope_free, self.rope)):
            f(h)


@pytest.mark.parametrize("M,sequences,f32", [(1, 1, True), (60, 60, False), (130, 2, True), (1000, 2, False), (2050, 1, True)])
@pytest.mark.parametrize("adapters", [True, False])
def test_one_call_is_the_calls_one_by_one_and_the_formula(M, sequences, f32, adapters):
    import torch
    b = Block(M, sequences, f32)
    st = torch.cuda.current_stream().cuda_stream
    b.one_call(b.y[0], st, adapters)
    b.one_by_one(b.y[1], st, adapters)
    torch.cuda.synchronize()
    assert B.lq_get_device_status(0)[0] == 0
    got = b.y[0].cpu().numpy()
    assert np.array_equal(got, b.y[1].cpu().numpy())
    if adapters:
        ref = b.formula()
        # the oracle's forward within 1e-5 of a row's size, the adapters and heads far below that; a norm divides by the row's size, so the
        # errors stay relative to the largest of a head.  fp16: Y is rounded between the calls (three times for queries and keys)
        tol = 4e-5 if f32 else 4 * 2.0 ** -11
        scale = np.abs(ref.reshape(M, -1, b.D)).max(-1, keepdims=True)
        err = np.abs(got.astype(np.float64) - ref).reshape(M, -1, b.D) / scale
        assert err.max() <= tol, err.max()
    b.free()


def test_captured_with_other_requests_on_each_replay():
    import torch
    b = Block(300, 2, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b.one_call(b.y[0], side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.one_call(b.y[0], torch.cuda.current_stream().cuda_stream)
    rng = np.random.default_rng(9)
    for _ in range(2):
        b.i.copy_(torch.from_numpy(rng.integers(-1, 2, 300).astype(np.int32)))
        b.x.copy_(torch.from_numpy(rng.standard_normal((300, b.K)).astype(np.float16)))
        b.p.copy_(torch.from_numpy(rng.integers(0, 100, (300, 2)).astype(np.int32)))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = b.y[0].clone()
        b.one_by_one(b.y[1], torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(want, b.y[1])
    del graph
    b.free()


def test_two_streams_with_maps_of_their_own():
    """The same layer's adapters on two streams at once, each with a map and buffers of its own."""
    import torch
    blocks = [Block(700, 1, False, seed=s) for s in (1, 2)]
    torch.cuda.synchronize()
    for b in blocks:
        b.one_by_one(b.y[1], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b.one_call(b.y[0], s.cuda_stream)
    torch.cuda.synchronize()
    for b in blocks:
        assert torch.equal(b.y[0], b.y[1])
        b.free()


def test_launches_without_overlap_give_the_same():
    import torch
    b = Block(900, 3, True)
    st = torch.cuda.current_stream().cuda_stream
    b.one_call(b.y[0], st)
    torch.cuda.synchronize()
    B.lq_set_option("overlap", 0)
    try:
        b.one_call(b.y[1], st)
        torch.cuda.synchronize()
    finally:
        B.lq_set_option("overlap", 1)
    assert torch.equal(b.y[0], b.y[1])
    b.free()


def test_refusals():
    import torch
    b = Block(64, 2, False)
    B.lq_rowmap_set(b.map, b.i.data_ptr(), 64, 0)
    torch.cuda.synchronize()
    b.y[0].fill_(3.0)

    def code(M=64, set_=b.set, map_=b.map, y=None, x=None, dtype=None, **q):
        c = B.lq_qkv(b.D, b.hq, b.hk, b.seqs, B.NORM_RMS, 1e-6, b.rope, b.p.data_ptr())
        for k, v in q.items():
            setattr(c, k, v)
        try:
            B.lq_qkv_forward(b.h, b.act, b.x.data_ptr() if x is None else x, M, set_, map_, c, b.y[0].data_ptr() if y is None else y, b.code if dtype is None else dtype, 0)
        except B.LqError as e:
            return e.code
        return 0

    assert code(set_=None) == 1 and code(map_=None) == 1 and code(M=62) == 1 and code(M=65) == 1 and code(M=0) == 1
    assert code(sequences=3) == 1 and code(sequences=0) == 1 and code(q_heads=5) == 1 and code(head_dim=36) == 1 and code(kv_heads=0) == 1
    assert code(norm=7) == 1 and code(eps=-1.0) == 1 and code(rope=None) == 1 and code(pos_dev=None) == 1 and code(dtype=2) == 1
    assert code(y=b.y[0].data_ptr() + 8) == 1 and code(x=b.x.data_ptr() + 2) == 1 and code(q_bias=b.wd.data_ptr()) == 1
    other = B.lq_adapters_create(b.K + 8, b.N, 16, 2, 0)
    assert code(set_=other) == 1
    B.lq_adapters_free(other)
    torch.cuda.synchronize()
    assert (b.y[0] == 3).all()                             # a refused call has launched nothing
    assert code() == 0 and code(set_=None, map_=None) == 0
    torch.cuda.synchronize()
    assert B.lq_get_device_status(0)[0] == 0
    b.free()


def test_inputs_that_share_memory_with_outputs_under_adapters():
    import torch
    b = Block(64, 2, False)
    B.lq_rowmap_set(b.map, b.i.data_ptr(), 64, 0)
    torch.cuda.synchronize()
    b.y[0].fill_(3.0)
    c = B.lq_qkv(b.D, b.hq, b.hk, b.seqs, B.NORM_RMS, 1e-6, b.rope, b.p.data_ptr())
    with pytest.raises(B.LqError) as e:
        B.lq_qkv_forward(b.h, b.act, b.y[0].data_ptr(), 64, b.set, b.map, c, b.y[0].data_ptr(), b.code, 0)
    assert e.value.code == 1
    torch.cuda.synchronize()
    assert (b.y[0] == 3).all()
    b.free()


@pytest.mark.parametrize("adapters", [True, False])
def test_weights_and_positions_among_the_values_are_refused(adapters):
    """The GEMM writes the values' columns too, before the heads read their weights and the rows' positions."""
    import torch
    b = Block(64, 2, False)
    B.lq_rowmap_set(b.map, b.i.data_ptr(), 64, 0)
    torch.cuda.synchronize()
    b.y[0].fill_(3.0)
    Y, v = b.y[0].data_ptr(), 2 * (b.hq + b.hk) * b.D      # the first row's values, 576 bytes of them
    end = Y + 2 * b.M * b.N

    def code(p=b.p.data_ptr(), q_weight=None, k_weight=None, norm=B.NORM_RMS, q_bias=None, k_bias=None):
        c = B.lq_qkv(b.D, b.hq, b.hk, b.seqs, norm, 1e-6, b.rope, p, q_weight, k_weight, q_bias, k_bias)
        try:
            B.lq_qkv_forward(b.h, b.act, b.x.data_ptr(), 64, b.set if adapters else None, b.map if adapters else None, c, Y, b.code, 0)
        except B.LqError as e:
            return e.code
        return 0

    assert code(p=Y + v) == 1 and code(p=end - 4) == 1 and code(p=Y - 64 * 2 * 4 + 4) == 1
    assert code(q_weight=Y + v) == 1 and code(k_weight=Y + v) == 1 and code(k_weight=end - 16) == 1
    assert code(norm=B.NORM_LAYER, q_bias=Y + v) == 1 and code(norm=B.NORM_LAYER, k_bias=Y + v) == 1
    torch.cuda.synchronize()
    assert (b.y[0] == 3).all()                             # a refused call has launched nothing
    assert code() == 0
    torch.cuda.synchronize()
    b.free()


def _within(b, got):
    ref, tol = b.formula(), 4e-5 if b.f32 else 4 * 2.0 ** -11          # as in the first test above
    scale = np.abs(ref.reshape(b.M, -1, b.D)).max(-1, keepdims=True)
    return (np.abs(got.astype(np.float64) - ref).reshape(b.M, -1, b.D) / scale).max() <= tol


@pytest.mark.parametrize("M,sequences,f32", [(60, 60, False), (130, 2, True), (1900, 1, False)])
def test_without_adapters_against_the_formula(M, sequences, f32):
    import torch
    b = Block(M, sequences, f32)
    b.one_call(b.y[0], torch.cuda.current_stream().cuda_stream, adapters=False)
    torch.cuda.synchronize()
    b.ids[:] = -1
    assert _within(b, b.y[0].cpu().numpy())
    b.free()


def test_one_layer_set_and_table_on_two_streams():
    """What a server has once for all its streams: layer, adapters and rotation.  Maps, activations and outputs are each stream's own; one stream has
    few rows, the other many."""
    import torch
    one, two = Block(300, 2, True, seed=1), Block(2050, 1, True, seed=2)
    for f, h in ((B.lq_act_free, two.act), (B.lq_layer_free, two.h), (B.lq_adapters_free, two.set), (B.lq_rope_free, two.rope)):
        f(h)
    two.layer, two.h, two.set, two.rope, two.A, two.Bf = one.layer, one.h, one.set, one.rope, one.A, one.Bf
    two.act = B.lq_act_create(two.h, two.M, 0)
    two.qkv = B.lq_qkv(two.D, two.hq, two.hk, two.seqs, B.NORM_RMS, 1e-6, two.rope, two.p.data_ptr(), two.wd[0].data_ptr(), two.wd[1].data_ptr())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for b in (one, two):
        b.one_by_one(b.y[1], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for turn in range(10):
        for b in (one, two):
            b.y[0].fill_(7)
        torch.cuda.synchronize()
        for _ in range(5):
            for b, s in zip((one, two), streams):
                b.one_call(b.y[0], s.cuda_stream)
        torch.cuda.synchronize()
        for b in (one, two):
            assert torch.equal(b.y[0], b.y[1]), turn
    for b in (one, two):
        assert _within(b, b.y[0].cpu().numpy())
    B.lq_act_free(two.act)
    B.lq_rowmap_free(two.map)
    one.free()


def test_a_refused_allocation_is_not_a_later_calls_error():
    """A set, or a record, that no GPU has room for is refused; the calls behind it are what they were."""
    import torch
    b = Block(64, 2, False)
    st = torch.cuda.current_stream().cuda_stream
    b.one_by_one(b.y[1], st)
    for create in (lambda: B.lq_adapters_create(8192, 1 << 20, 128, 1023, 0), lambda: B.lq_act_create(b.h, 1 << 30, 0)):
        with pytest.raises(B.LqError) as e:
            create()
        assert e.value.code == 3
        b.one_call(b.y[0], st)
        torch.cuda.synchronize()
        assert torch.equal(b.y[0], b.y[1])
    b.free()
