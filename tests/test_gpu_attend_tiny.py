"""spf_attend on 8-bit caches where the factor from products to logits leaves fp32's range: tiny queries over keys of the smallest scale
(zeros, as spf_kv_append writes them), huge ones over keys of the largest.  Keys that a row does not see stay out of its sums."""
import pytest
import torch

from attend_reference import check, gpu_step
from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,new", [(2, 1, 64, 1), (2, 1, 128, 1), (4, 1, 64, 4), (4, 1, 64, 8), (4, 1, 64, 40), (4, 1, 128, 40)])
@pytest.mark.parametrize("query,key", [(-30, -100), (-45, -100), (-100, -100), (-126, -100), (100, 100), (126, 100)])
def test_factors_beyond_the_range(Hq, Hkv, d, new, query, key):
    """Logits of zero, by zero keys, times a factor of about 2^(query + key): the mean of the values that a row sees."""
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 128, [300], [new], 8, seed=query + 200)
    s.k_pool.zero_()
    s.k_scale.fill_(2.0 ** key)
    s.q.clamp_(-2, 2).mul_(2.0 ** (query - 1))
    out, lse = run(spf, s)
    check(s, out, lse)
    out, lse = run(spf, s, first=[130])                     # and masked at both ends
    check(s, out, lse, first=[130])
