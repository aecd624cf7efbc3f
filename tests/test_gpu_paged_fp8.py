"""spf_score_paged_fp8 (8-bit block pools with a scale for each 64 tokens of a block and head) against the oracle on the decoded
keys: their values, E4M3 times a power of two, are bf16 numbers."""
import numpy as np
import pytest
import torch

import oracle
from kv_reference import e4m3_values
from workloads import bf16_bits, make_prompt, small_config

pytestmark = pytest.mark.gpu


def make_pools(k_layers, n, block, seed, spread=2):
    """8-bit pools with shuffled blocks whose groups of 64 tokens have scales of their own, and the decoded keys as bf16
    [Hkv, N, d].  What no token of the prompt lies in holds NaN bytes and NaN scales."""
    g = torch.Generator().manual_seed(seed)
    n_blocks = -(-n // block)
    perm = torch.randperm(n_blocks + 2, generator=g)[:n_blocks].to(torch.int32)
    pools, scales, decoded = [], [], []
    for k in k_layers:
        Hkv, _, d = k.shape
        x = torch.zeros((Hkv, n_blocks * block, d))
        x[:, :n] = k.float().cpu()
        x = x.view(Hkv, -1, 64, d) * 2.0 ** torch.randint(-spread, spread + 1, (Hkv, n_blocks * block // 64, 1, 1), generator=g).float()
        s = 2.0 ** torch.ceil(torch.log2(x.abs().amax((-1, -2)).clamp(min=2.0 ** -40) / 448.0))
        raw = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        values = (e4m3_values(raw) * s.double()[..., None, None]).view(Hkv, -1, d)[:, :n]
        decoded.append(values.to(torch.bfloat16))
        assert torch.equal(decoded[-1].double(), values)
        raw = raw.view(Hkv, -1, d)
        raw[:, n:] = 0x7F
        s[:, -(-n // 64):] = float("nan")
        pool = torch.full((n_blocks + 2, Hkv, block, d), 0x7F, dtype=torch.uint8)
        scale = torch.full((n_blocks + 2, Hkv, block // 64), float("nan"))
        for b in range(n_blocks):
            pool[perm[b]] = raw[:, b * block:(b + 1) * block]
            scale[perm[b]] = s[:, b * block // 64:(b + 1) * block // 64]
        pools.append(pool.cuda())
        scales.append(scale.cuda())
    return pools, scales, perm.cuda(), decoded


CASES = [
    # L, Hq, Hkv, d, m, N, block
    (2, 8, 2, 64, 8, 20000, 4096),
    (2, 4, 2, 128, 8, 9001, 1024),
    (1, 4, 1, 64, 16, 30000, 128),
    (1, 2, 1, 64, 8, 100, 256),
    (3, 4, 1, 128, 16, 5000, 384),
    (1, 5, 1, 64, 3, 777, 128),
    (2, 2, 2, 128, 1, 64, 128),
    (1, 1, 1, 64, 2, 1, 128),
]


def _prompt(L, Hq, Hkv, d, m, N, block):
    cfg = small_config("paged8", n_layers=L, n_q_heads=Hq, n_kv_heads=Hkv, head_dim=d, n_lookahead=m, lengths=(N,), rank=4,
                       n_needles=2 if N >= 300 else 0, n_strong=1, needle_len=(4, 40), seed=N + block)
    prompt = make_prompt(cfg, 0, "cpu")
    prompt.q.mul_(0.5)      # groups' magnitudes differ by up to 4: logits stay where exp's argument is a number of two digits
    return prompt


def _score(spf, prompts, path, extra_rows=0):
    outer = spf.spf_set_score_path(path)
    try:
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(spf.spf_score_paged_fp8_workspace_bytes(prompts), dtype=torch.uint8, device="cuda")
        spf.spf_score_paged_fp8(prompts, ws, 0.0, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
    finally:
        spf.spf_set_score_path(outer)


@pytest.mark.parametrize("path", [0, 1])
@pytest.mark.parametrize("L,Hq,Hkv,d,m,N,block", CASES)
def test_scoring(L, Hq, Hkv, d, m, N, block, path):
    import paper_2603_02631_b200 as spf
    prompt = _prompt(L, Hq, Hkv, d, m, N, block)
    pools, scales, table, decoded = make_pools(prompt.k, N, block, seed=N)
    want, want_lse = oracle.token_importance(bf16_bits(prompt.q), [bf16_bits(x) for x in decoded])
    imp = torch.empty(N, device="cuda")
    lse = torch.empty((L, Hq, m), device="cuda")
    _score(spf, [spf.PagedFp8PromptBuffers(prompt.q.cuda(), pools, scales, table, N, imp, lse)], path)
    got = imp.cpu().numpy()
    assert np.isfinite(got).all()
    assert np.max(np.abs(got - want) / np.maximum(want, 1e-30)) <= 1e-3
    assert np.allclose(lse.cpu().numpy().ravel(), np.asarray(want_lse).ravel(), rtol=1e-4, atol=1e-4)


@pytest.mark.parametrize("path", [0, 1])
def test_batch_of_prompts(path):
    import paper_2603_02631_b200 as spf
    lens, bufs, wants = (3000, 129, 9000), [], []
    for i, n in enumerate(lens):
        prompt = _prompt(2, 8, 2, 64, 8, n, 256)
        pools, scales, table, decoded = make_pools(prompt.k, n, 256, seed=i)
        wants.append(oracle.token_importance(bf16_bits(prompt.q), [bf16_bits(x) for x in decoded])[0])
        bufs.append(spf.PagedFp8PromptBuffers(prompt.q.cuda(), pools, scales, table, n, torch.empty(n, device="cuda")))
    _score(spf, bufs, path)
    for b, want in zip(bufs, wants):
        got = b.importance.cpu().numpy()
        assert np.max(np.abs(got - want) / np.maximum(want, 1e-30)) <= 1e-3


def test_selector():
    """Selector.run_paged_fp8 gives what the calls one by one give."""
    import paper_2603_02631_b200 as spf
    L, Hq, Hkv, d, m, N, block = 2, 8, 2, 64, 8, 5000, 256
    prompt = _prompt(L, Hq, Hkv, d, m, N, block)
    pools, scales, table, _ = make_pools(prompt.k, N, block, seed=1)
    dp = prompt.to("cuda:0")
    imp = torch.empty(N, device="cuda")
    _score(spf, [spf.PagedFp8PromptBuffers(dp.q, pools, scales, table, N, imp)], 0)
    sel = spf.Selector(L, Hq, Hkv, d, m, N)
    got = sel.run_paged_fp8(dp.q, pools, scales, table, N, dp.token_ids, dp.char_start, dp.char_end, 0.25)
    torch.cuda.synchronize()
    assert int(sel.dev_status.item()) == 0
    assert torch.equal(got.importance, imp)
    scores = torch.empty((N + 31) // 32, device="cuda")
    kept = torch.empty(got.k, dtype=torch.int32, device="cuda")
    spf.spf_chunk_pool(imp, 13, 32, scores)
    spf.spf_select_topk(scores, scores.numel(), got.k, kept)
    torch.cuda.synchronize()
    assert torch.equal(kept, got.kept_chunks[:got.k])
    with pytest.raises(ValueError):
        sel.run_paged_fp8(dp.q, pools, scales[:1], table, N, dp.token_ids, dp.char_start, dp.char_end, 0.25)
    with pytest.raises(TypeError):
        sel.run_paged_fp8(dp.q, pools, [s.double() for s in scales], table, N, dp.token_ids, dp.char_start, dp.char_end, 0.25)
    with pytest.raises(ValueError):
        spf.spf_score_paged_fp8_workspace_bytes([spf.PagedFp8PromptBuffers(dp.q, pools, [s[:, :, :1] for s in scales], table, N, imp)])
