"""spf_score_paged_fp8 on prompts of more than 32 key tiles a CTA, whose scales are fetched in several goes."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_paged_fp8 import _prompt, _score, make_pools
from workloads import bf16_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", [1, 2])               # the general kernels, and the fused one: 33 to 35 tiles on each of 148 SMs
@pytest.mark.parametrize("Hq,d,m,N", [(2, 64, 8, 650001), (4, 64, 8, 640123), (8, 64, 2, 625000), (2, 128, 4, 650001)])
def test_a_prompt_of_many_tiles_a_cta(Hq, d, m, N, path):
    import paper_2603_02631_b200 as spf
    prompt = _prompt(1, Hq, 1, d, m, N, 4096)
    pools, scales, table, decoded = make_pools(prompt.k, N, 4096, seed=N)
    want, want_lse = oracle.token_importance(bf16_bits(prompt.q), [bf16_bits(x) for x in decoded])
    imp, lse = torch.empty(N, device="cuda"), torch.empty((1, Hq, m), device="cuda")
    _score(spf, [spf.PagedFp8PromptBuffers(prompt.q.cuda(), pools, scales, table, N, imp, lse)], path)
    got = imp.cpu().numpy()
    assert np.max(np.abs(got - want) / np.maximum(want, 1e-30)) <= 1e-3
    assert np.allclose(lse.cpu().numpy().ravel(), np.asarray(want_lse).ravel(), rtol=1e-4, atol=1e-4)
