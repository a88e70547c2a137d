"""Attention where a few tokens outweigh each of very many: what the many weigh together counts beside the values as it does in the sum."""
import numpy as np
import pytest

from paper_2604_18117_b200 import binding as B

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def run(D, sequences, tokens, heavy, rows, gap, causal=False):
    """`heavy` first tokens of value 0 that weigh e^gap each, the others 1, of value 64 (beside an entry that tells the sequences apart)."""
    import torch
    pages = -(-tokens // 64)
    c = B.lq_kvcache_create(1, sequences * pages, 64, 1, D)
    order = torch.from_numpy(np.random.default_rng(3).permutation(sequences * pages).astype(np.int32).reshape(sequences, pages)).cuda()
    k = torch.zeros(sequences, tokens, 1, D, dtype=torch.float16, device="cuda")
    k[:, :heavy, :, 0] = gap                               # (whole halves: codes of a step of 1/4)
    v = torch.full_like(k, 64.0)
    v[..., 1] = torch.arange(1, sequences + 1, device="cuda").view(-1, 1, 1) % 16 + 48
    v[:, :heavy] = 0
    length = torch.full((sequences,), tokens, dtype=torch.int32, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    kr = B.lq_kvrows(k.data_ptr(), (0, D, D), v.data_ptr(), (0, D, D))
    B.lq_kvcache_append(c, 0, B.lq_kvbatch(sequences, sequences * tokens, length.data_ptr(), order.data_ptr(), pages), kr, B.OUT_F16, st)
    q = torch.zeros(sequences * rows, 1, D, dtype=torch.float16, device="cuda")
    q[..., 0] = 1
    out = torch.empty_like(q)
    B.lq_cache_attention(c, 0, B.lq_kvbatch(sequences, sequences * rows, length.data_ptr(), order.data_ptr(), pages),
                         B.lq_attn(q.data_ptr(), (D, D), out.data_ptr(), (D, D), 1, 1.0, causal), st)
    got = out.view(sequences, rows, D).double().cpu().numpy()
    light = tokens - heavy
    total = heavy + light * np.exp(-gap)
    value = v[:, -1, 0].double().cpu().numpy()[:, None]
    want = light * np.exp(-gap) * value / total
    # A weight is rounded to a half of up to 2^15 (2^7 and 8 powers of two that the maximum may run ahead): to 2^-11 of it, or, where it is below 2^-14, by
    # 2^-25, which is 2^-32 of the weight of the reference; no reference is more than 2^8 below the largest (then small weights only keep more).  The
    # exponent is exact here but for scale times log2 e and the power: 2 u of it, and 8 u.  Sums: 2 sqrt(n) + 64 roundings.
    err = (2.0 ** -11 + (4 * gap + 2 * np.sqrt(tokens) + 64) * U) * want + light * 2.0 ** -32 * value / total
    err = err + (want + err) * 2.0 ** -11 + 2.0 ** -25
    far = np.abs(got - want) / err
    assert far.max() <= 1, (float(far.max()), got[0, 0, :2], want[0, 0, :2])
    B.lq_kvcache_free(c)


@pytest.mark.parametrize("gap", [12.0, 15.0, 16.5, 17.0, 17.5, 18.0])
@pytest.mark.parametrize("D", [64, 128])
def test_a_prompt(D, gap):
    """Tiles of rows that one thread block takes through the whole sequence."""
    run(D, 1, 20000, 1, 40000, gap)


@pytest.mark.parametrize("gap", [15.0, 17.0, 17.5])
def test_a_prompt_that_is_shared_out(gap):
    run(64, 1, 100000, 1, 200, gap)


@pytest.mark.parametrize("gap", [12.0, 15.0, 16.5, 17.0, 17.5, 18.0])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_single_tokens(D, gap):
    """More tiles than thread blocks; a heavy token in the first record of each warp of one."""
    run(D, 600, 3000, 256, 1, gap)


def test_one_long_sequence():
    run(128, 1, 100000, 4096, 1, 17.0)
