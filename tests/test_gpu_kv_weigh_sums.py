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
