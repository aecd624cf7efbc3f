"""spf_attend over caches of 4 bits against the 64-bit reference: single tokens, a few, many; masks that leave rows empty."""
import math

import pytest
import torch

from kv4_reference import attention4, compare4, make_step4

pytestmark = pytest.mark.gpu


def run(spf, s, causal=True, first=None, scale=0.0, max_new=None, lse_heads_outside=False, status=0):
    out = torch.full((s.rows, s.Hq, s.d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((s.Hq, s.rows), 7.0, device="cuda").T if lse_heads_outside else torch.full((s.rows, s.Hq), 7.0, device="cuda")
    seen = torch.zeros(1, dtype=torch.int32, device="cuda")
    step = s.step(spf, max_new)
    workspace = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), step, s.q), dtype=torch.uint8, device="cuda")
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    spf.spf_attend(s.cache(spf), step, s.q, out, workspace, lse, f, causal, scale, seen)
    torch.cuda.synchronize()
    assert int(seen.item()) == status
    return out, lse


CASES = [
    # Hq, Hkv, d, block, tokens before, new tokens
    (4, 2, 64, 128, [0], [1]),                              # one key
    (8, 8, 128, 128, [63, 64, 65, 127, 128, 0], [1] * 6),   # around tiles' and blocks' ends, every head its own keys
    (16, 2, 128, 256, [1000], [1]),                         # one sequence over many CTAs
    (10, 2, 64, 384, [700, 0, 129], [1, 0, 1]),             # five heads a group, a sequence without new tokens
    (32, 8, 64, 1024, [800, 30], [8, 3]),                   # lookahead tokens: 32 rows
    (8, 1, 128, 128, [300, 70], [2, 1]),                    # 16 rows
    (8, 1, 128, 128, [300, 70], [8, 2]),                    # 64 rows
    (3, 1, 64, 128, [100], [5]),                            # 15 rows
    (5, 1, 128, 256, [400], [40]),                          # 200 rows
    (8, 2, 64, 128, [0, 250], [130, 70]),                   # a prompt from its first token on
    (6, 2, 128, 128, [0, 511], [400, 129]),                 # two tiles of 256 rows, several tiles of keys
]


@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", CASES)
def test_attention(Hq, Hkv, d, block, old, new):
    import paper_2603_02631_b200 as spf
    s = make_step4(Hq, Hkv, d, block, old, new, seed=d + block + len(old), behind=2)
    compare4(s, *run(spf, s))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("max_new", [1, 4, 16, 1000])
def test_the_hint_changes_nothing_but_the_kernels(d, max_new):
    import paper_2603_02631_b200 as spf
    s = make_step4(8, 2, d, 128, [200, 3, 500], [6, 1, 20], seed=max_new, fused=False)
    compare4(s, *run(spf, s, max_new=max_new, lse_heads_outside=True))


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [4, 9, 2, 30]])
def test_first_keys_that_leave_rows_empty_and_rows_that_see_all(new):
    import paper_2603_02631_b200 as spf
    s = make_step4(6, 2, 64, 128, [150, 63, 400, 128], new, seed=3, behind=1)
    first = [150, 64, -5, 1000]                             # its own tokens; all but the first; all; none
    for causal in (True, False):
        compare4(s, *run(spf, s, causal=causal, first=first, scale=0.2), causal=causal, first=first, scale=0.2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [1, 6, 90])
def test_what_no_row_may_see_does_not_matter(new, d):
    """Scales that are not finite, and other codes, behind the sequence, before its first key and in other sequences' blocks."""
    import paper_2603_02631_b200 as spf
    old, first = [230, 80], [70, 3]
    s = make_step4(8, 2, d, 128, old, [new, new], seed=4)
    clean = run(spf, s, first=first)
    used = torch.zeros(s.k_pool.shape[:1] + s.k_pool.shape[2:3], dtype=torch.bool)
    for b in range(2):
        for pos in range(first[b], old[b] + new):
            used[int(s.table[b, pos // 128]), pos % 128] = True
    unused = ~used.cuda()[:, None, :, None]
    for name in ("k_scale", "v_scale", "k_pool", "v_pool"):
        held = getattr(s, name)
        for value in (float("nan"), float("inf"), -3e38) if "scale" in name else (0, 255):
            keep = held.clone()
            held.masked_fill_(unused, value)
            dirty = run(spf, s, first=first)
            assert torch.equal(clean[0], dirty[0]) and torch.equal(clean[1], dirty[1]), (name, value)
            held.copy_(keep)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("new", [6, 100])
def test_values_that_are_nan_reach_the_rows_that_see_them_and_no_others(new, d):
    import paper_2603_02631_b200 as spf
    s = make_step4(4, 2, d, 128, [90], [new], seed=5)
    clean, lse = run(spf, s)
    at = 90 + new // 2                                      # a token of the step
    s.v_scale[int(s.table[0, at // 128]), 0, at % 128, 1] = float("nan")
    out, same = run(spf, s)
    assert torch.equal(lse, same)
    assert torch.isnan(out[new // 2:, :2, 32:64]).all()
    assert torch.equal(out[:new // 2], clean[:new // 2])
    rest = torch.ones(out.shape, dtype=torch.bool)
    rest[:, :2, 32:64] = False
    assert torch.equal(out.cpu()[rest], clean.cpu()[rest])


def test_queries_that_are_not_finite_and_very_different_ones():
    import paper_2603_02631_b200 as spf
    s = make_step4(4, 1, 64, 128, [300], [2], seed=6)
    clean, clean_lse = run(spf, s)
    q = s.q.clone()
    s.q = q.clone()
    s.q[0, 1, 5], s.q[0, 2, 7] = float("nan"), float("inf")
    out, lse = run(spf, s)
    assert torch.isnan(out[0, 1:3]).all() and torch.isnan(lse[0, 1:3]).all()
    assert torch.equal(out[1], clean[1]) and torch.equal(out[0, 0], clean[0, 0]) and torch.equal(out[0, 3], clean[0, 3])
    for power in (-90, -20, 40, 110):                       # of all elements, with the softmax scale that undoes it
        s.q = (q.float() * 2.0 ** power).to(torch.bfloat16)
        scale = 0.125 * 2.0 ** -power
        compare4(s, *run(spf, s, scale=scale), scale=scale)
    s.q = q.clone()
    s.q[:, :, ::2] *= 2.0 ** -30                            # elements far apart in a row
    compare4(s, *run(spf, s))


@pytest.mark.parametrize("new", [1, 80])
def test_steep_softmax_and_scales_far_apart(new):
    import paper_2603_02631_b200 as spf
    s = make_step4(4, 1, 64, 128, [900], [new], seed=6)
    compare4(s, *run(spf, s, scale=3.0), scale=3.0)
    gen = torch.Generator().manual_seed(1)
    s.v_scale.copy_((2.0 ** torch.randint(-40, 31, s.v_scale.shape, generator=gen).float()).to(torch.bfloat16))
    compare4(s, *run(spf, s))
    s.v_scale.fill_(2.0 ** -40)
    compare4(s, *run(spf, s))
    s.v_scale.fill_(2.0 ** 50)
    compare4(s, *run(spf, s))
    s.k_scale.mul_(2.0 ** -60)
    compare4(s, *run(spf, s, scale=2.0 ** 57), scale=2.0 ** 57)


@pytest.mark.parametrize("what", ["block", "negative block", "length", "short"])
@pytest.mark.parametrize("new", [1, 100])
def test_bad_blocks_and_lengths_are_reported(what, new):
    import paper_2603_02631_b200 as spf
    s = make_step4(2, 1, 64, 128, [200, 300], [new, new], seed=8)
    if what == "block":
        s.table[1, 1] = s.k_pool.shape[0]
    elif what == "negative block":
        s.table[1, 0] = -3
    elif what == "length":
        s.seq_lens[1] = 128 * s.table.shape[1] + 1
    else:
        s.seq_lens[1] = 0
    out, lse = run(spf, s, status=-7)
    compare4(s, out, lse, seqs=[0])                         # the other sequence is not affected
    if what == "short":
        assert (out[new:] == 0).all() and (lse[new:] == -math.inf).all()


def test_graph_replayed_with_other_lengths():
    import paper_2603_02631_b200 as spf
    s = make_step4(8, 2, 128, 128, [1000, 100, 700], [1, 1, 1], seed=9)
    spare = [b for b in range(s.k_pool.shape[0]) if b not in s.table.flatten().tolist()]
    s.table[1, 1] = spare[0]
    step = s.step(spf)
    ws = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), step, s.q), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(s.q).contiguous(), torch.zeros((3, 8), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spf.spf_attend(s.cache(spf), step, s.q, out, ws, lse)
    for lens in ([1001, 101, 701], [1000, 129, 3], [64, 1, 700]):
        s.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        s.old = [n - 1 for n in lens]
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        compare4(s, out, lse)


def test_the_same_bits_every_time_and_random_steps():
    import random
    import paper_2603_02631_b200 as spf
    rng = random.Random(11)
    for i in range(25):
        d, Hkv, group = rng.choice([64, 128]), rng.choice([1, 2, 3]), rng.choice([1, 2, 3, 4, 8, 16])
        seqs = rng.randint(1, 4)
        new = [rng.choice([0, 1, 1, 2, 5, 17, 40]) for _ in range(seqs)]
        old = [rng.choice([0, 1, 31, 64, 127, 128, 129, 400]) for _ in range(seqs)]
        s = make_step4(group * Hkv, Hkv, d, rng.choice([128, 256]), old, new, seed=i, behind=rng.randint(0, 2), fused=rng.random() < 0.5)
        causal = rng.random() < 0.8
        first = [rng.randint(0, 200) for _ in range(seqs)] if rng.random() < 0.4 else None
        hint = rng.choice([None, 1, 9, 300])
        a, b = run(spf, s, causal, first, max_new=hint), run(spf, s, causal, first, max_new=hint)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        compare4(s, *a, causal=causal, first=first)


def test_large_pool_beyond_32_bit_offsets():
    """Blocks whose bytes lie behind 2^32."""
    import paper_2603_02631_b200 as spf
    n_blocks, Hkv, block, d = 6000, 8, 4096, 64
    s = make_step4(16, 8, d, block, [900], [1], seed=10)
    k_pool = torch.zeros((n_blocks, Hkv, block, d // 2), dtype=torch.uint8, device="cuda")
    scale = torch.ones((n_blocks, Hkv, block, d // 32), dtype=torch.bfloat16, device="cuda")
    k_pool[n_blocks - 1], scale[n_blocks - 1] = s.k_pool[int(s.table[0, 0])], s.k_scale[int(s.table[0, 0])]
    s.k_pool = s.v_pool = k_pool
    s.k_scale = s.v_scale = scale
    s.table = torch.tensor([[n_blocks - 1]], dtype=torch.int32, device="cuda")
    out, lse = run(spf, s)
    small = make_step4(16, 8, d, block, [900], [1], seed=10)
    small.v_pool, small.v_scale = small.k_pool, small.k_scale
    compare4(small, out, lse)
    assert attention4(small, 0)[0].shape == (1, 16, d)
