"""The draft model's side of the path as a serving loop runs it: two prompts appended layer by layer and attended over, lookahead
tokens one by one, whose rotated queries go straight to where the scoring calls read them, then importance and selection from the
same pools.  Each stage against the 64-bit references, on what the stages before it left."""
import math

import numpy as np
import pytest
import torch

import oracle
from kv_reference import attention, logical, rope_table, rotate
from workloads import bf16_bits

pytestmark = pytest.mark.gpu

L, HQ, HKV, D, M, BLOCK = 2, 8, 2, 64, 4, 512
PROMPTS = (300, 131)


def _check_rows(out, lse, q, cache, table_row, pos, operand):
    k, v = logical(cache.k_pool, cache.k_scale, table_row, pos[-1] + 1), logical(cache.v_pool, cache.v_scale, table_row, pos[-1] + 1)
    want, want_lse, weight, terms = attention(q, k, v, pos)
    off = terms * 2.0 ** -16 + 2.0 ** -20                  # as derived for spf_attend's own tests
    assert ((lse.double().cpu() - want_lse).abs() <= off + 2.0 ** -22 * want_lse.abs()).all()
    bound = 2.0 ** -8 * want.abs() + (operand + 2 * off[..., None]) * weight * (1 + 2.0 ** -8)
    assert ((out.double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_draft_model_prompt_lookahead_scoring(bits):
    import paper_2603_02631_b200 as spf
    gen = torch.Generator().manual_seed(bits)
    B, operand = len(PROMPTS), 2.0 ** -8 if bits == 16 else 2.0 ** -11
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    kind = torch.bfloat16 if bits == 16 else torch.uint8
    scale = lambda: None if bits == 16 else new(5, HKV, BLOCK // 64, dtype=torch.float32)  # noqa: E731
    caches = [spf.KvCache(new(5, HKV, BLOCK, D, dtype=kind), new(5, HKV, BLOCK, D, dtype=kind), scale(), scale()) for _ in range(L)]
    table = torch.tensor([[3], [1]], dtype=torch.int32, device="cuda")
    rope = rope_table(BLOCK, D)
    r = spf.Rope(rope.cuda())
    status = new(1, dtype=torch.int32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    # the prompts, both in one step
    rows = sum(PROMPTS)
    step = spf.KvStep(i32([0, PROMPTS[0], rows]), i32(PROMPTS), table, max(PROMPTS))
    workspace = new(spf.spf_attend_workspace_bytes(caches[0], step, new(rows, HQ, D)), dtype=torch.uint8)
    for cache in caches:
        qkv = torch.randn((rows, HQ + 2 * HKV, D), generator=gen).to(torch.bfloat16).cuda()
        q, out, lse = new(rows, HQ, D), new(rows, HQ, D), new(rows, HQ, dtype=torch.float32)
        spf.spf_kv_append(cache, step, qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], qkv[:, :HQ], q, r, status)
        spf.spf_attend(cache, step, q, out, workspace, lse, dev_status=status)
        torch.cuda.synchronize()
        turned, bound = rotate(qkv[:, :HQ], rope, torch.cat([torch.arange(n) for n in PROMPTS]))
        assert ((q.double().cpu() - turned).abs() <= 2.0 ** -8 * turned.abs() + 2 * bound).all()
        for b in range(B):
            part = slice(int(step.row_start[b]), int(step.row_start[b]) + PROMPTS[b])
            _check_rows(out[part], lse[part], q[part], cache, table[b], list(range(PROMPTS[b])), operand)

    # lookahead tokens: queries into [prompt][L][Hq][m][d], log-sum-exps into [prompt][L][Hq][m]
    queries, all_keys, own_keys = new(B, L, HQ, M, D), new(B, L, HQ, M, dtype=torch.float32), new(B, L, HQ, M, dtype=torch.float32)
    first = i32(PROMPTS)
    for i in range(M):
        step = spf.KvStep(i32(list(range(B + 1))), i32([n + i + 1 for n in PROMPTS]), table, 1)
        for l, cache in enumerate(caches):
            qkv = (torch.randn((B, HQ + 2 * HKV, D), generator=gen) * 1.5).to(torch.bfloat16).cuda()
            q, out = queries[:, l, :, i], new(B, HQ, D)
            spf.spf_kv_append(cache, step, qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], qkv[:, :HQ], q, r, status)
            spf.spf_attend(cache, step, q, out, workspace, all_keys[:, l, :, i], dev_status=status)
            spf.spf_attend(cache, step, q, new(B, HQ, D), workspace, own_keys[:, l, :, i], first_keys=first, dev_status=status)
            torch.cuda.synchronize()
            for b, n in enumerate(PROMPTS):
                _check_rows(out[b:b + 1], all_keys[b:b + 1, l, :, i], q[b:b + 1], cache, table[b], [n + i], operand)
    assert int(status.item()) == 0

    # importance and selection from the same pools
    for b, n in enumerate(PROMPTS):
        keys = [logical(c.k_pool, c.k_scale, table[b], n).to(torch.bfloat16) for c in caches]      # exact: bf16, or E4M3 times 2^e
        ids = torch.arange(n, dtype=torch.int32, device="cuda")
        sel = spf.Selector(L, HQ, HKV, D, M, n)
        args = (ids, ids * 2, ids * 2 + 2, 0.25)
        if bits == 16:
            got = sel.run_paged(queries[b], [c.k_pool for c in caches], table[b], n, *args)
        else:
            got = sel.run_paged_fp8(queries[b], [c.k_pool for c in caches], [c.k_scale for c in caches], table[b], n, *args)
        torch.cuda.synchronize()
        assert int(sel.dev_status.item()) == 0
        want, want_lse = oracle.token_importance(bf16_bits(queries[b].cpu()), [bf16_bits(x) for x in keys])
        imp = got.importance.cpu().numpy()
        assert np.max(np.abs(imp - want) / np.maximum(want, 1e-30)) <= 1e-3
        kept = oracle.select_topk(got.chunk_scores.double().cpu().numpy(), got.k)
        assert got.kept_chunks[:got.k].cpu().tolist() == kept.tolist()
        # a lookahead row's keys are the prompt's and its own: exp(all) = exp(prompt) + exp(own), each off by its own bound
        joined = np.logaddexp(want_lse, own_keys[b].double().cpu().numpy())
        assert np.abs(joined - all_keys[b].double().cpu().numpy()).max() <= 1e-3
        if bits == 16:
            # the prompt lies in one block: the same keys as a contiguous cache, with the own keys in the denominator
            imp2 = new(n, dtype=torch.float32)
            bufs = spf.PromptBuffers(queries[b].contiguous(), [c.k_pool[int(table[b, 0]), :, :n] for c in caches], imp2)
            ws = new(spf.spf_score_workspace_bytes([bufs]), dtype=torch.uint8)
            spf.spf_score_extra([bufs], [own_keys[b].contiguous()], ws, 0.0, status)
            torch.cuda.synchronize()
            want2, _ = oracle.token_importance(bf16_bits(queries[b].cpu()), [bf16_bits(x) for x in keys],
                                               extra_lse=own_keys[b].double().cpu().numpy())
            assert np.max(np.abs(imp2.cpu().numpy() - want2) / np.maximum(want2, 1e-30)) <= 1e-3
    assert int(status.item()) == 0


@pytest.mark.parametrize("bits", [16, 8])
def test_a_lookahead_step_as_a_graph(bits):
    """Append and attention of one token captured once and replayed for token after token, as a decoding loop does: lengths live on
    the device, new projections are written in place."""
    import paper_2603_02631_b200 as spf
    gen = torch.Generator().manual_seed(3)
    kind = torch.bfloat16 if bits == 16 else torch.uint8
    pools = [torch.zeros((4, HKV, 128, D), dtype=kind, device="cuda") for _ in range(2)]
    scales = [None if bits == 16 else torch.zeros((4, HKV, 2), device="cuda") for _ in range(2)]
    cache = spf.KvCache(*pools, *scales)
    table = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
    lens, starts = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    step, rope = spf.KvStep(starts, lens, table, 1), rope_table(400, D)
    qkv = torch.zeros((1, HQ + 2 * HKV, D), dtype=torch.bfloat16, device="cuda")
    q, out, lse = torch.zeros((1, HQ, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, HQ, D), dtype=torch.bfloat16, device="cuda"), \
        torch.zeros((1, HQ), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = spf.Rope(rope.cuda())
    ws = torch.empty(spf.spf_attend_workspace_bytes(cache, step, q), dtype=torch.uint8, device="cuda")
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        lens += 1
        spf.spf_kv_append(cache, step, qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], qkv[:, :HQ], q, r, status)
        spf.spf_attend(cache, step, q, out, ws, lse, dev_status=status)
    lens.zero_()
    for t in range(140):
        qkv.copy_(torch.randn(qkv.shape, generator=gen).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        if t in (0, 1, 63, 64, 127, 128, 139):
            _check_rows(out, lse, q, cache, table[0], [t], 2.0 ** -8 if bits == 16 else 2.0 ** -11)
    assert int(status.item()) == 0 and int(lens.item()) == 140
