"""spf_kv_weigh against the 64-bit reference: caches of 16, 8 and 4 bits, few and many rows, masks, decay, positions."""
import math

import pytest
import torch

from ledger_reference import any_step, ledger_of, received

pytestmark = pytest.mark.gpu


def weigh(spf, s, lse, weight, position, status=0, first=None, max_new=None, **settings):
    seen = torch.zeros(1, dtype=torch.int32, device="cuda")
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    spf.spf_kv_weigh(s.cache(spf), s.step(spf, max_new), s.q, lse, spf.KvLedger(weight, position), first_keys=f, dev_status=seen, **settings)
    torch.cuda.synchronize()
    assert int(seen.item()) == status


def reference_lse(s, bits, first=None, causal=True, scale=None, outside=False):
    lse = torch.zeros((s.rows, s.Hq))
    for b, new in enumerate(s.new):
        if new:
            lse[int(s.row_start[b]):int(s.row_start[b]) + new] = received(s, bits, b, 0 if first is None else max(first[b], 0), causal, scale)[2]
    return lse.T.contiguous().cuda().T if outside else lse.cuda()


def check(spf, s, bits, first=None, causal=True, scale=None, last=0, decay=1.0, positions=None, max_new=None, with_position=True, outside=False):
    lse = reference_lse(s, bits, first, causal, scale, outside)
    weight, position = ledger_of(s, 5, with_position)
    before, places = weight.cpu().double(), None if position is None else position.cpu()
    weigh(spf, s, lse, weight, position, first=first, max_new=max_new, causal=causal, softmax_scale=scale or 0.0, last_rows=last, decay=decay,
          positions=None if positions is None else positions.cuda())
    want, slack = before.clone(), torch.zeros_like(before)
    for b, (old, new) in enumerate(zip(s.old, s.new)):
        if new == 0:
            continue
        n, row = old + new, int(s.row_start[b])
        got, off, _ = received(s, bits, b, 0 if first is None else max(first[b], 0), causal, scale, last, lse)
        key = torch.arange(n)
        at, place = s.table.cpu()[b][key // s.block].long(), key % s.block
        held = torch.where(key[:, None] < old, want[at, :, place] * decay, torch.zeros(1, dtype=torch.float64))
        want[at, :, place] = held + got.T
        slack[at, :, place] = off.T + 2.0 ** -22 * (held + got.T)
        if places is not None:
            new_at = positions[row:row + new] if positions is not None else torch.arange(old, n, dtype=torch.int32)
            places[at[old:], :, place[old:]] = new_at[:, None].expand(-1, s.Hkv)
    off = (weight.cpu().double() - want).abs() - slack
    assert (off <= 0).all(), float(off.max())
    if position is not None:
        assert torch.equal(position.cpu(), places)


CASES = [
    # Hq, Hkv, d, block, tokens before, new tokens
    (4, 2, 64, 128, [0], [1]),
    (8, 8, 128, 128, [63, 64, 65, 127, 128, 0], [1] * 6),
    (16, 2, 128, 256, [1000], [1]),
    (10, 2, 64, 384, [700, 0, 129], [1, 0, 1]),
    (32, 8, 64, 1024, [800, 30], [8, 3]),
    (8, 1, 128, 128, [300, 70], [2, 1]),
    (3, 1, 64, 128, [100], [5]),
    (5, 1, 128, 256, [400], [40]),
    (8, 2, 64, 128, [0, 250], [130, 70]),
    (6, 2, 128, 128, [0, 511], [300, 129]),
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", CASES)
def test_received_weights(Hq, Hkv, d, block, old, new, bits):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, Hq, Hkv, d, block, old, new, d + block + len(old), behind=2)
    check(spf, s, bits, decay=0.75)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("max_new", [1, 4, 16, 1000])
def test_the_hint_changes_nothing_but_the_kernels(bits, max_new):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, 8, 2, 128, 128, [200, 3, 500], [6, 1, 20], max_new, fused=False)
    check(spf, s, bits, max_new=max_new, outside=True, with_position=False)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [4, 9, 2, 70]])
def test_masks_last_rows_and_positions(bits, new):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, 6, 2, 64, 128, [150, 63, 400, 128], new, 3, behind=1)
    first = [150, 64, -5, 1000]
    positions = torch.randint(0, 9999, (s.rows,), generator=torch.Generator().manual_seed(2)).to(torch.int32)
    for causal in (True, False):
        for last in (0, 1, 3, 50):
            check(spf, s, bits, first, causal, 0.2, last, 0.0 if last == 1 else 0.5, positions)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [1, 7, 90])
def test_rows_that_are_not_numbers_and_keys_that_no_row_sees(bits, new):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, 4, 2, 64, 128, [200], [new], 4)
    lse = reference_lse(s, bits)
    clean = ledger_of(s, 5)[0]
    weigh(spf, s, lse, clean, None)
    # what lies behind the sequence does not matter
    block, place = int(s.table[0, (200 + new) // 128]) if (200 + new) // 128 < s.table.shape[1] else None, (200 + new) % 128
    if block is not None:
        if bits == 4:
            s.k_scale[block, :, place:] = float("nan")
        else:
            s.k_pool[block, :, place:] = float("nan") if bits == 16 else 0x7F
    again = ledger_of(s, 5)[0]
    weigh(spf, s, lse, again, None)
    assert torch.equal(clean, again)
    # a row whose log-sum-exp is -inf adds nothing, one with NaN makes NaN of what it sees, in its own head
    lse[new - 1, 0], lse[new // 2, 3] = -math.inf, float("nan")
    odd = ledger_of(s, 5)[0]
    weigh(spf, s, lse, odd, None)
    key = torch.arange(200 + new)
    at, place = s.table.cpu()[0][key // 128].long(), key % 128
    got, was = odd.cpu()[at, :, place], clean.cpu()[at, :, place]
    assert torch.isnan(got[:200 + new // 2 + 1, 1]).all() and torch.equal(got[200 + new // 2 + 1:, 1], was[200 + new // 2 + 1:, 1])
    assert torch.isfinite(got[:, 0]).all() and (got[:, 0] <= was[:, 0]).all() and (got[:100, 0] < was[:100, 0]).any()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("what", ["block", "negative block", "length", "short"])
def test_bad_blocks_and_lengths_are_reported(bits, what):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, 2, 1, 64, 128, [200, 300], [1, 1], 8)
    lse = reference_lse(s, bits)
    good, _ = ledger_of(s, 5)
    weigh(spf, s, lse, good, None)
    gone = int(s.table[1, 1])
    if what == "block":
        s.table[1, 1] = s.k_pool.shape[0]
    elif what == "negative block":
        s.table[1, 1] = -3
    elif what == "length":
        s.seq_lens[1] = 128 * s.table.shape[1] + 1
    else:
        s.seq_lens[1] = 0
    got, position = ledger_of(s, 5)
    before = got.clone()
    weigh(spf, s, lse, got, position, status=-7)
    key = torch.arange(201)
    at, place = s.table.cpu()[0][key // 128].long(), key % 128
    assert torch.equal(got.cpu()[at, :, place], good.cpu()[at, :, place])           # the other sequence is not affected
    if "block" in what:
        assert torch.equal(got[gone], before[gone])


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_graph_replayed_with_other_lengths_and_the_same_bits_every_time(bits):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, 8, 2, 128, 128, [1000, 100, 700], [1, 1, 1], 9)
    lse = torch.zeros((3, 8), device="cuda")
    weight, position = ledger_of(s, 5)
    start = weight.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spf.spf_kv_weigh(s.cache(spf), s.step(spf), s.q, lse, spf.KvLedger(weight, position), decay=0.5)
    for lens in ([1001, 101, 701], [900, 128, 3], [64, 1, 700]):
        s.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        s.old = [n - 1 for n in lens]
        lse.copy_(reference_lse(s, bits))
        weight.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        other = start.clone()
        weigh(spf, s, lse, other, None, decay=0.5)
        assert torch.equal(weight, other)
        check(spf, s, bits, decay=0.5)


def test_random_steps():
    import random
    import paper_2603_02631_b200 as spf
    rng = random.Random(12)
    for i in range(45):
        bits, d, Hkv, group = rng.choice([16, 8, 4]), rng.choice([64, 128]), rng.choice([1, 2, 3]), rng.choice([1, 2, 3, 4, 8, 16])
        seqs = rng.randint(1, 4)
        new = [rng.choice([0, 1, 1, 2, 5, 17, 40]) for _ in range(seqs)]
        old = [rng.choice([0, 1, 31, 64, 127, 128, 129, 400]) for _ in range(seqs)]
        s = any_step(bits, group * Hkv, Hkv, d, rng.choice([128, 256]), old, new, i, behind=rng.randint(0, 2), fused=rng.random() < 0.5)
        first = [rng.randint(0, 200) for _ in range(seqs)] if rng.random() < 0.4 else None
        check(spf, s, bits, first, rng.random() < 0.8, None, rng.choice([0, 0, 1, 4, 16]), rng.choice([0.0, 0.9, 1.0]), None, rng.choice([None, 1, 9, 300]))
