"""spf_kv_append to caches of 4 bits with enough rows for the variant that has a warp to a token, at both head dimensions."""
import copy

import pytest
import torch

from kv4_reference import make_step4
from kv_reference import rope_table
from test_gpu_kv4_append import append, check
from test_gpu_kv_append_wide import enough

pytestmark = pytest.mark.gpu

NAMES = ("k_pool", "v_pool", "k_scale", "v_scale")


def few_for(Hq, Hkv, d):
    """Tokens that are half of what the variant is taken from."""
    return 148 * 2048 // ((Hq + 2 * Hkv) * d // 16) // 2


@pytest.mark.parametrize("Hq,Hkv,d,rot_dim,interleaved,given", [
    (6, 3, 128, 128, False, False), (7, 7, 128, 32, True, True), (24, 12, 128, 128, True, False), (5, 5, 64, 32, False, True), (9, 3, 64, 64, True, True),
    (1, 1, 128, 96, False, True), (1, 1, 64, 64, False, False), (16, 2, 64, 48, False, False), (33, 11, 128, 80, True, True), (8, 8, 64, 64, False, True),
])
def test_many_rows(Hq, Hkv, d, rot_dim, interleaved, given):
    import paper_2603_02631_b200 as spf
    few = few_for(Hq, Hkv, d)
    s = make_step4(Hq, Hkv, d, 384, [70, 0, 1000, 5], [few + 77, few, 0, 63], seed=Hq + d, behind=3)
    assert enough(s)
    positions = torch.randint(0, 9000, (s.rows,), generator=torch.Generator().manual_seed(2)).to(torch.int32) if given else None
    check(spf, s, rope_table(max(9000, 2 * few + 200), rot_dim), positions, interleaved)


@pytest.mark.parametrize("d", [64, 128])
def test_without_rotation_without_queries_and_heads_outside(d):
    import paper_2603_02631_b200 as spf
    shape = (8, 4, d, 256, [100, 0], [3000, 1900])
    s = make_step4(*shape, seed=1, fused=False)
    assert enough(s)
    check(spf, s)
    check(spf, make_step4(*shape, seed=2), rope_table(3200, 64), with_q=False)
    check(spf, make_step4(*shape, seed=3), with_q=False)
    check(spf, make_step4(*shape, seed=4, fused=False), rope_table(3200, 32), interleaved=True)


@pytest.mark.parametrize("Hq,Hkv,d,rot_dim,interleaved", [(8, 4, 64, 64, False), (5, 3, 128, 128, False), (5, 3, 128, 64, True), (12, 2, 64, 0, False)])
def test_the_bytes_are_those_of_few_rows_and_of_queries_in_place(Hq, Hkv, d, rot_dim, interleaved):
    """Against the variant for few rows, which is given the same tokens in parts; zeros, infinities and NaN among them."""
    import paper_2603_02631_b200 as spf
    few = few_for(Hq, Hkv, d)
    whole = make_step4(Hq, Hkv, d, 256, [100, 0, 37], [few + 60, 1, few], seed=9)
    assert enough(whole)
    inf, nan = float("inf"), float("nan")
    for x in (whole.k, whole.v):
        x[3], x[5, 0, 7], x[5, -1, 40], x[6, 0, 3], x[7] = 0, inf, -inf, nan, -inf
        x[8, 0], x[9, 0] = 3.3e38, 2.0 ** -130
    parts, placed = copy.deepcopy(whole), copy.deepcopy(whole)
    table = rope_table(few + 200, rot_dim) if rot_dim else None
    q = append(spf, whole, table, None, interleaved)
    rope = None if table is None else spf.Rope(table.cuda(), None, interleaved)
    spf.spf_kv_append(placed.cache(spf), placed.step(spf), placed.k, placed.v, placed.q, placed.q, rope)
    q_parts, at_once = torch.zeros_like(q), few // 3
    for b, (old, new) in enumerate(zip(whole.old, whole.new)):
        for done in range(0, new, at_once):
            n, row = min(at_once, new - done), int(whole.row_start[b]) + done
            i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
            step = spf.KvStep(i32([0, n]), i32([old + done + n]), whole.table[b:b + 1].contiguous(), n)
            rows = slice(row, row + n)
            spf.spf_kv_append(parts.cache(spf), step, parts.k[rows], parts.v[rows], parts.q[rows], q_parts[rows], rope)
    torch.cuda.synchronize()
    for x in NAMES:
        for other in (parts, placed):
            assert torch.equal(getattr(whole, x).view(torch.uint8), getattr(other, x).view(torch.uint8)), x
    assert torch.equal(q, q_parts) and torch.equal(q, placed.q)


@pytest.mark.parametrize("what", ["block", "position", "short"])
def test_places_outside_are_reported_and_left_out(what):
    import paper_2603_02631_b200 as spf
    s = make_step4(8, 4, 64, 256, [100, 0], [3000, 1900], seed=5)
    assert enough(s)
    positions = torch.arange(s.rows, dtype=torch.int32) % 3000
    good = copy.deepcopy(s)
    q_good = append(spf, good, rope_table(3200, 64), positions)
    before = {x: getattr(s, x).clone() for x in NAMES}
    out = torch.zeros(s.rows, dtype=torch.bool)              # rows that are left out
    gone = torch.zeros(s.k_pool.shape[:1] + s.k_pool.shape[2:3], dtype=torch.bool)
    blocks, table = s.k_pool.shape[0], s.table.cpu()
    if what == "block":
        out[156:412] = True                                  # places 256 to 511 of the first sequence
        gone[int(table[0, 1])] = True
        s.table[0, 1] = blocks
    elif what == "position":
        for row, value in ((7, -1), (2500, 3200), (3001, 2 ** 31 - 1)):
            positions[row], out[row] = value, True
            place = 100 + row if row < 3000 else row - 3000
            gone[int(table[int(row >= 3000), place // 256]), place % 256] = True
    else:
        s.seq_lens[1] = 1200                                 # 1900 tokens, the first 700 of which are before place 0
        out[3000:3700] = True
        gone[table[1][table[1] >= 0].long()] = True
    q = append(spf, s, rope_table(3200, 64), positions, status=-7)
    assert (q[out] == 7).all() and not (q[~out] == 7).all(-1).any()
    assert torch.equal(q[~out], q_good[~out])
    for x in NAMES:
        got, want, was = (t.transpose(1, 2).cpu() for t in (getattr(s, x), getattr(good, x), before[x]))
        assert torch.equal(got[~gone].view(torch.uint8), want[~gone].view(torch.uint8)), x
        if what != "short":
            assert torch.equal(got[gone].view(torch.uint8), was[gone].view(torch.uint8)), x
