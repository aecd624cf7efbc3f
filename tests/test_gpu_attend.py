"""spf_attend against the 64-bit reference: single tokens, a few, many; bf16 and 8-bit pools; masks that leave rows empty."""
import math

import pytest
import torch

from kv_reference import attention, logical, make_step

pytestmark = pytest.mark.gpu


def run(spf, s, causal=True, first=None, scale=0.0, max_new=None, lse_heads_outside=False, workspace=None):
    out = torch.full((s.rows, s.Hq, s.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((s.Hq, s.rows) if lse_heads_outside else (s.rows, s.Hq), 7.0, device="cuda")
    lse = lse.T if lse_heads_outside else lse
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    step = s.step(spf, max_new)
    if workspace is None:
        workspace = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), step, s.q), dtype=torch.uint8, device="cuda")
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    spf.spf_attend(s.cache(spf), step, s.q, out, workspace, lse, f, causal, scale, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out, lse


def compare(s, out, lse, causal=True, first=None, scale=None, seqs=None):
    """Tolerances.  A logit is an fp32 sum of d exact products (both factors have at most 11 bits): off by at most
    d 2^-24 sum |q k|, which is below 2^-16 sum with the scaling's roundings; the weights are off by that twice (the sum has it
    too), by ex2's 2^-21, and by half a step of the second product's operands (bf16 2^-8, fp16 2^-11); the output by half a step
    of bf16."""
    operand = 2.0 ** -8 if s.k_scale is None else 2.0 ** -11
    for b, (old, new) in enumerate(zip(s.old, s.new)):
        if new == 0 or (seqs is not None and b not in seqs):
            continue
        start = int(s.row_start[b])
        rows = slice(start, start + new)
        k, v = logical(s.k_pool, s.k_scale, s.table[b], old + new), logical(s.v_pool, s.v_scale, s.table[b], old + new)
        want, want_lse, weight, terms = attention(s.q[rows], k, v, range(old, old + new), 0 if first is None else max(first[b], 0), causal, scale)
        off = terms * 2.0 ** -16 + 2.0 ** -20
        got, got_lse = out[rows].double().cpu(), lse[rows].double().cpu()
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(got_lse) & (got_lse < 0), empty)
        assert (got[empty] == 0).all()
        seen = ~empty
        assert ((got_lse - want_lse)[seen].abs() <= off[seen] + 2.0 ** -22 * want_lse[seen].abs()).all()
        bound = 2.0 ** -8 * want.abs() + (operand + 2 * off[..., None]) * weight * (1 + 2.0 ** -8)
        assert ((got - want).abs() <= bound).all(), float(((got - want).abs() - bound).max())
    rows = sum(s.new)
    assert (out[rows:] == 7.0).all() and (lse[rows:] == 7.0).all()


CASES = [
    # Hq, Hkv, d, block, tokens before, new tokens
    (4, 2, 64, 128, [0], [1]),                              # one key
    (8, 8, 128, 128, [63, 64, 65, 127, 128, 0], [1] * 6),   # around tiles' and blocks' ends, every head its own keys
    (16, 2, 128, 256, [1000], [1]),                         # one sequence over many CTAs
    (10, 2, 64, 384, [700, 0, 129], [1, 0, 1]),             # five heads a group, a sequence without new tokens
    (32, 8, 64, 1024, [1500, 30], [8, 3]),                  # lookahead tokens: 32 rows
    (8, 1, 128, 128, [300, 70], [8, 2]),                    # 64 rows
    (3, 1, 64, 128, [100], [5]),                            # 15 rows
    (5, 1, 128, 256, [400], [40]),                          # 200 rows
    (8, 2, 64, 128, [0, 250], [130, 70]),                   # a prompt from its first token on
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", CASES)
def test_attention(Hq, Hkv, d, block, old, new, bits):
    import paper_2603_02631_b200 as spf
    s = make_step(Hq, Hkv, d, block, old, new, bits, seed=d + block + len(old), behind=2)
    out, lse = run(spf, s)
    compare(s, out, lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("max_new", [1, 4, 16, 1000])
def test_the_hint_changes_nothing_but_the_kernels(bits, max_new):
    import paper_2603_02631_b200 as spf
    s = make_step(8, 2, 128, 128, [200, 3, 500], [6, 1, 20], bits, seed=max_new, fused=False)
    out, lse = run(spf, s, max_new=max_new, lse_heads_outside=True)
    compare(s, out, lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [4, 9, 2, 30]])
def test_first_keys_that_leave_rows_empty_and_rows_that_see_all(bits, new):
    import paper_2603_02631_b200 as spf
    old = [150, 63, 400, 128]
    s = make_step(6, 2, 64, 128, old, new, bits, seed=3, behind=1)
    first = [150, 64, -5, 1000]                             # its own tokens; all but the first; all; none
    for causal in (True, False):
        out, lse = run(spf, s, causal=causal, first=first, scale=0.2)
        compare(s, out, lse, causal=causal, first=first, scale=0.2)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [1, 6, 90])
def test_what_no_row_may_see_does_not_matter(bits, new):
    """NaN and infinities in the pool behind the sequence, before its first key and in other sequences' blocks."""
    import paper_2603_02631_b200 as spf
    old, first = [230, 80], [70, 3]
    s = make_step(8, 2, 64, 128, old, [new, new], bits, seed=4)
    clean = run(spf, s, first=first)
    bad = [float("nan"), float("inf"), float("-inf")] if bits == 16 else [0x7F, 0xFF]
    used = torch.zeros(s.k_pool.shape[:1] + s.k_pool.shape[2:3], dtype=torch.bool)
    for b in range(2):
        for pos in range(first[b], old[b] + new):
            used[int(s.table[b, pos // 128]), pos % 128] = True
    for pool in (s.k_pool, s.v_pool):
        for value in bad:
            keep = pool.clone()
            pool.masked_fill_(~used.cuda()[:, None, :, None], value)
            dirty = run(spf, s, first=first)
            assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[1], dirty[1])
            pool.copy_(keep)


@pytest.mark.parametrize("new", [1, 6, 90])
def test_scales_of_groups_that_no_row_sees_do_not_matter(new):
    import paper_2603_02631_b200 as spf
    old, first = [230, 80], [70, 3]                         # the group of tokens 0 to 63 of the first is seen by nobody
    s = make_step(8, 2, 64, 128, old, [new, new], 8, seed=4)
    clean = run(spf, s, first=first)
    used = torch.zeros(s.k_scale.shape[:1] + s.k_scale.shape[2:], dtype=torch.bool)
    for b in range(2):
        for pos in range(first[b], old[b] + new):
            used[int(s.table[b, pos // 128]), pos % 128 // 64] = True
    for scale in (s.k_scale, s.v_scale):
        for value in (0.0, float("nan"), float("inf"), -1.0):
            keep = scale.clone()
            scale.masked_fill_(~used.cuda()[:, None], value)
            dirty = run(spf, s, first=first)
            assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[1], dirty[1])
            scale.copy_(keep)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [6, 100])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_and_no_others(bits, new):
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, 64, 128, [90], [new], bits, seed=5)
    clean, lse = run(spf, s)
    at = 90 + new // 2                                      # a token of the step
    block = int(s.table[0, at // 128])
    s.v_pool[block, 0, at % 128, 3] = float("nan") if bits == 16 else 0x7F
    if bits == 16:
        s.v_pool[block, 1, at % 128, 60] = float("inf")
    out, same = run(spf, s)
    assert torch.equal(lse, same)
    got = out.float().cpu()
    assert torch.isnan(got[new // 2:, :2, 3]).all()
    if bits == 16:
        assert torch.isinf(got[new // 2:, 2:, 60]).all()
    assert torch.equal(out[:new // 2], clean[:new // 2])
    rest = torch.ones_like(got, dtype=torch.bool)
    rest[:, :2, 3] = False
    rest[:, 2:, 60] = False
    assert torch.isfinite(got[rest]).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_steep_softmax_and_scales_far_apart(bits):
    """One key far above the rest, growing logits along the keys, and value scales from 2^-30 to 2^30."""
    import paper_2603_02631_b200 as spf
    s = make_step(4, 1, 64, 128, [999], [1], bits, seed=6)
    out, lse = run(spf, s, scale=3.0)
    compare(s, out, lse, scale=3.0)
    if bits == 8:
        s.v_scale.copy_(2.0 ** torch.randint(-30, 31, s.v_scale.shape, generator=torch.Generator().manual_seed(1)).float())
        s.k_scale *= 3.0                                    # not a power of two
        out, lse = run(spf, s)
        compare(s, out, lse)
        s.q.mul_(2.0 ** -20)
        out, lse = run(spf, s, scale=2.0 ** 17)
        compare(s, out, lse, scale=2.0 ** 17)


@pytest.mark.parametrize("bits", [16, 8])
def test_many_sequences(bits):
    import paper_2603_02631_b200 as spf
    old = [(37 * b) % 200 for b in range(400)]
    new = [(b % 5 != 3) * 1 for b in range(400)]
    s = make_step(2, 1, 64, 128, old, new, bits, seed=7)
    out, lse = run(spf, s)
    compare(s, out, lse, seqs=list(range(0, 400, 7)))


@pytest.mark.parametrize("bits", [16, 8])
def test_bad_blocks_and_lengths_are_reported(bits):
    import paper_2603_02631_b200 as spf
    for what in ("block", "negative block", "length", "short"):
        s = make_step(2, 1, 64, 128, [200, 300], [1, 1], bits, seed=8)
        if what == "block":
            s.table[1, 1] = s.k_pool.shape[0]
        elif what == "negative block":
            s.table[1, 0] = -3
        elif what == "length":
            s.seq_lens[1] = 128 * s.table.shape[1] + 1
        else:
            s.seq_lens[1] = 0
        out = torch.full((2, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), s.step(spf), s.q), dtype=torch.uint8, device="cuda")
        lse = torch.zeros((2, 2), device="cuda")
        spf.spf_attend(s.cache(spf), s.step(spf), s.q, out, ws, lse, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == -7, what
        lens = s.old[0] + 1
        k, v = logical(s.k_pool, s.k_scale, s.table[0], lens), logical(s.v_pool, s.v_scale, s.table[0], lens)
        want, _, weight, _ = attention(s.q[:1], k, v, [200])
        assert ((out[:1].double().cpu() - want).abs() <= 2.0 ** -6 * weight).all()          # the other sequence is not affected
        if what == "short":
            assert (out[1] == 0).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_graph_replayed_with_other_lengths_two_graphs_on_one_workspace_and_another_stream(bits):
    import paper_2603_02631_b200 as spf
    s = make_step(8, 2, 64, 128, [1200, 100, 700], [1, 1, 1], bits, seed=9)
    spare = [b for b in range(s.k_pool.shape[0]) if b not in s.table.flatten().tolist()]
    s.table[1, 1] = spare[0]                                # the second sequence grows to 129 tokens below
    step = s.step(spf)
    ws = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), step, s.q), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros_like(s.q).contiguous() for _ in range(2)]
    lses = [torch.zeros((3, 8), device="cuda") for _ in range(2)]
    stream, graphs = torch.cuda.Stream(), []
    stream.wait_stream(torch.cuda.current_stream())
    for out, lse, causal in zip(outs, lses, (True, False)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            spf.spf_attend(s.cache(spf), step, s.q, out, ws, lse, causal=causal)
        graphs.append(graph)
    for lens in ([1201, 101, 701], [1000, 129, 3], [64, 1, 700]):
        s.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        s.old = [n - 1 for n in lens]
        ws.fill_(255)                                       # whatever the workspace holds
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for out, lse in zip(outs, lses):
            compare(s, out, lse)
    with torch.cuda.stream(stream):
        again = torch.zeros_like(outs[0])
        spf.spf_attend(s.cache(spf), step, s.q, again, ws, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(again, outs[0])


def test_large_pool_beyond_32_bit_offsets():
    """Blocks whose bytes lie behind 2^32."""
    import paper_2603_02631_b200 as spf
    n_blocks, Hkv, block, d = 6000, 8, 4096, 64             # 12.6e9 elements of 8 bits
    k_pool = torch.zeros((n_blocks, Hkv, block, d), dtype=torch.uint8, device="cuda")
    scale = torch.ones((n_blocks, Hkv, block // 64), device="cuda")
    s = make_step(16, 8, 64, block, [5000], [1], 8, seed=10)
    table = torch.tensor([[n_blocks - 1, n_blocks - 2]], dtype=torch.int32, device="cuda")
    for j in range(2):
        k_pool[n_blocks - 1 - j] = s.k_pool[int(s.table[0, j])]
        scale[n_blocks - 1 - j] = s.k_scale[int(s.table[0, j])]
    s.k_pool = s.v_pool = k_pool
    s.k_scale = s.v_scale = scale
    s.table = table
    out, lse = run(spf, s)
    compare(s, out, lse)
