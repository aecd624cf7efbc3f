"""Calls on the draft model's cache that are allowed and rarely made: wide groups of heads, steps without tokens, shared blocks, garbage
behind the sequences' table entries, two calls at once, repeated calls."""
import pytest
import torch

from kv_reference import make_step, rope_table
from test_gpu_attend import compare, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,old,new", [(33, 1, 64, [150, 3], [1, 1]), (64, 1, 128, [500], [1]), (40, 1, 64, [130], [7]), (16, 2, 128, [300, 40], [3, 2]), (12, 12, 128, [70], [300])])
def test_wide_groups_and_single_heads(Hq, Hkv, d, old, new, bits):
    """33, 64, 280 and 24 rows of a key head (the kernel for many rows, few tokens); one row a head of a prompt."""
    import paper_2603_02631_b200 as spf
    s = make_step(Hq, Hkv, d, 128, old, new, bits, seed=Hq, behind=1)
    compare(s, *run(spf, s))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("max_new", [1, 100])
def test_a_step_in_which_no_sequence_has_tokens(bits, max_new):
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, 64, 128, [100, 0, 300], [0, 0, 0], bits, seed=1, behind=3)
    before = [x.clone() for x in (s.k_pool, s.v_pool)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full_like(s.q, 7.0)
    spf.spf_kv_append(s.cache(spf), s.step(spf, max_new), s.k, s.v, s.q, q_out, spf.Rope(rope_table(400, 64).cuda()), status)
    out, lse = run(spf, s, max_new=max_new)
    assert (out == 7.0).all() and (lse == 7.0).all() and (q_out == 7.0).all() and int(status.item()) == 0
    assert all(torch.equal(a, b) for a, b in zip(before, (s.k_pool, s.v_pool)))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d,new", [(64, 6), (128, 2), (64, 60), (128, 60)])
def test_queries_that_are_not_finite_spoil_their_own_row_alone(d, new, what, bits):
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, d, 128, [300], [new], bits, seed=8)
    clean, clean_lse = run(spf, s)
    element = s.q[1, 2, 5].clone()
    s.q[1, 2, 5] = what
    out, lse = run(spf, s)
    assert out[1, 2].isnan().all() and lse[1, 2].isnan()
    s.q[1, 2, 5] = element                                  # the other rows: as the reference has them
    out[1, 2], lse[1, 2] = clean[1, 2], clean_lse[1, 2]
    compare(s, out, lse)


def test_a_step_of_no_rows():
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, 64, 128, [100], [0], 16, seed=2)
    assert s.rows == 0
    spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q, torch.empty_like(s.q))
    run(spf, s)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [1, 50])
def test_sequences_that_share_blocks_and_entries_behind_their_ends(bits, new):
    """The same blocks twice give the same rows; table entries behind a sequence's length may hold anything."""
    import paper_2603_02631_b200 as spf
    s = make_step(8, 2, 128, 128, [300, 300], [new, new], bits, seed=3)
    s.table[1] = s.table[0]
    s.table = torch.cat([s.table, torch.full((2, 2), 1 << 30, dtype=torch.int32, device="cuda")], 1).contiguous()
    s.q[new:2 * new] = s.q[:new]
    out, lse = run(spf, s)
    compare(s, out, lse)
    # parts of the two are cut at other keys, so that sums differ in their last bits; the reference bounds both
    again, lse_again = run(spf, s)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("bits", [16, 8])
def test_two_calls_at_once(bits):
    """Two streams, each with a workspace of its own; few rows beside many."""
    import paper_2603_02631_b200 as spf
    steps = [make_step(16, 4, 64, 128, [9000], [1], bits, seed=4), make_step(8, 2, 128, 128, [700], [400], bits, seed=5)]
    alone = [run(spf, s) for s in steps]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs, spaces, lses = [], [], []
    for s in steps:
        outs.append(torch.zeros((s.rows, s.Hq, s.d), dtype=torch.bfloat16, device="cuda"))
        lses.append(torch.zeros((s.rows, s.Hq), device="cuda"))
        spaces.append(torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), s.step(spf), s.q), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(10):
        for s, out, lse, ws, stream in zip(steps, outs, lses, spaces, streams):
            spf.spf_attend(s.cache(spf), s.step(spf), s.q, out, ws, lse, stream=stream)
    torch.cuda.synchronize()
    for (out, lse), got, got_lse in zip(alone, outs, lses):
        assert torch.equal(out, got) and torch.equal(lse, got_lse)


@pytest.mark.parametrize("bits", [16, 8])
def test_append_twice_leaves_the_same_cache(bits):
    """A step that is run again on the cache it has written (a retried call): the same bytes and scales."""
    import paper_2603_02631_b200 as spf
    s = make_step(8, 4, 64, 128, [70, 5], [30, 200], bits, seed=6)
    table, out = rope_table(400, 64).cuda(), torch.empty_like(s.q)
    states = []
    for _ in range(2):
        spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q, out, spf.Rope(table))
        torch.cuda.synchronize()
        states.append([x.clone() for x in (s.k_pool, s.v_pool, s.k_scale, s.v_scale, out) if x is not None])
    assert all(torch.equal(a, b) for a, b in zip(*states))
