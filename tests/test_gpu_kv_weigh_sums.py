"""How near spf_kv_weigh comes to 64 bits: sums over thousands of rows, whatever the hint, and whole sets of weights, step by step and chunk by chunk."""
import math

import pytest
import torch

from test_gpu_kv4_long import decoded, gpu_step4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("max_new,one_row", [(1, False), (2, False), (4, False), (2000, False), (2000, True)])
def test_thousands_of_equal_weights(bits, max_new, one_row):
    """2000 tokens of 8 heads give every key the weight e^-L each (queries are zero).  L log2(e) is rounded twice, which moves a weight by 1.5 * 2^-24 *
    10.1 * ln 2 = 6.3e-7 at L = 7, ex2 by 2^-22; the 128 weights of a tile at most are added in fp32, four sums of 32: at most 16.5 * 2^-24 = 9.9e-7;
    what joins tiles, lanes and sets of warps a few times 2^-24.  All below 2^-18.  Added one tile after the other with what the additions lose
    left out, 2000 tiles of 8 rows are off by 1.6e-5 to 2.6e-5 at these L (counted out in numpy).  one_row: a row stride of zero, which the kernel for
    many rows does not take."""
    import paper_2603_02631_b200 as spf
    s = gpu_step4(32, 4, 64, 128, [60], [2000], bits, seed=1)
    s.q.zero_()
    lse = torch.tensor([1.5, 2.5, 5.5, 7.0], device="cuda").repeat_interleave(8).expand(2000, 32).contiguous()
    weight = torch.zeros(s.k_pool.shape[:3], device="cuda")
    spf.spf_kv_weigh(s.cache(spf), s.step(spf, max_new), s.q[:1].expand_as(s.q) if one_row else s.q, lse, spf.KvLedger(weight), causal=False)
    key = torch.arange(2060, device="cuda")
    got = weight[s.table[0].long()[key // 128], :, key % 128].double()
    want = 16000 * torch.exp(-lse[0, ::8].double())
    assert ((got / want - 1).abs() <= 2.0 ** -18).all(), float((got / want - 1).abs().max())


STEPS = [(16, 8, 128, 4096, [9000] * 6, [1] * 6), (32, 8, 64, 1024, [20000], [1]), (32, 8, 64, 1024, [20000], [8])]
CHUNKS = [(8, 2, 64, 4096, [3000, 0], [900, 700]), (3, 1, 128, 512, [9000], [513])]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", STEPS + CHUNKS)
def test_weights_of_long_sequences_in_the_2_norm(Hq, Hkv, d, block, old, new, bits):
    """The largest weights, which decide, belong to logits of 4 to 5.  Such a logit is the sum of d / 16 products' sums, each rounded off by 0.29 of a
    step on average, of up to 2^-23 of what is summed up so far: sqrt(3) * 0.29 * 1.4 * 2^-23 * 5 = 4.2e-7.  The exponent's rounding (0.29 * 2^-23 * 7
    ln 2) and ex2 (half of its 2^-22 at most) make 4.7e-7 of it, one key with another: below 6e-7.  Products of 8-bit keys with 8-bit queries would
    leave 1.3e-6, sums over thousands of rows without what the additions lose 1.7e-6."""
    import paper_2603_02631_b200 as spf
    s = gpu_step4(Hq, Hkv, d, block, old, new, bits, seed=d + bits, q_scale=0.5 if bits == 8 else 1.0)
    group, lse = Hq // Hkv, torch.zeros((s.rows, Hq), device="cuda")           # any number will do; 0 is not rounded on its way
    weight = torch.zeros(s.k_pool.shape[:3], device="cuda")
    spf.spf_kv_weigh(s.cache(spf), s.step(spf), s.q, lse, spf.KvLedger(weight))
    off, size = 0.0, 0.0
    for b, (o, n_new) in enumerate(zip(old, new)):
        n, row = o + n_new, int(s.row_start[b])
        key = torch.arange(n, device="cuda")
        hidden = key[None, :] > (o + torch.arange(n_new, device="cuda"))[:, None]
        at, place = s.table[b].long()[key // block], key % block
        for h in range(Hkv):
            k, want = decoded(s, bits, "k", b, h, n)[0], torch.zeros(n, dtype=torch.float64, device="cuda")
            for g in range(h * group, (h + 1) * group):
                want += torch.exp((s.q[row:row + n_new, g].double() @ k.T / math.sqrt(d)).masked_fill_(hidden, -math.inf)).sum(0)
            off += float((weight[at, h, place].double() - want).square().sum())
            size += float(want.square().sum())
    assert math.sqrt(off / size) <= 6e-7, math.sqrt(off / size)
