"""spf_kv_append to caches of 4 bits against the 64-bit reference: codes, scales, rotated queries, everything else untouched."""
import pytest
import torch

from kv4_reference import SCALE_DIMS, make_step4, short_scale, values
from kv_reference import rope_table, rotate

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8


def append(spf, s, rope=None, positions=None, interleaved=False, with_q=True, status=0):
    q_out = torch.full((s.rows, s.Hq, s.d), 7.0, dtype=torch.bfloat16, device="cuda")
    seen = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = None if rope is None else spf.Rope(rope.cuda(), None if positions is None else positions.cuda(), interleaved)
    spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q if with_q else None, q_out if with_q else None, r, seen)
    torch.cuda.synchronize()
    assert int(seen.item()) == status
    return q_out


def check(spf, s, rope=None, positions=None, interleaved=False, with_q=True):
    names = ("k_pool", "v_pool", "k_scale", "v_scale")
    before = {x: getattr(s, x).clone() for x in names}
    q_out = append(spf, s, rope, positions, interleaved, with_q)
    touched = torch.zeros(s.k_pool.shape[:1] + s.k_pool.shape[2:3], dtype=torch.bool)
    for b, (old, new) in enumerate(zip(s.old, s.new)):
        if new == 0:
            continue
        rows, pos = slice(int(s.row_start[b]), int(s.row_start[b]) + new), torch.arange(old, old + new)
        at = pos if positions is None else positions[rows].long()
        blocks, place = s.table.cpu()[b][pos // s.block].long(), pos % s.block
        touched[blocks, place] = True
        for x in "qkv":
            if x == "q" and not with_q:
                continue
            data = getattr(s, x)[rows]
            want, off = rotate(data, rope, at, interleaved) if rope is not None and x != "v" else (data.double().cpu(), torch.zeros(data.shape, dtype=torch.float64))
            if x == "q":
                assert ((q_out[rows].double().cpu() - want).abs() <= BF16 * want.abs() + 2 * off).all()
                continue
            scale = getattr(s, x + "_scale").cpu()[blocks, :, place].double()
            amax, slack = want.unflatten(-1, (-1, SCALE_DIMS)).abs().amax(-1), off.unflatten(-1, (-1, SCALE_DIMS)).amax(-1)
            assert (7 * scale >= amax - slack).all()
            for a, o, got in list(zip(amax.flatten().tolist(), slack.flatten().tolist(), scale.flatten().tolist()))[:500]:
                assert short_scale(a - o) <= got <= short_scale(a + o)
            # half a code, and what two roundings of the quotient (2^-23 of at most 7) and the rotation's may move
            got = values(getattr(s, x + "_pool").cpu()[blocks, :, place], getattr(s, x + "_scale").cpu()[blocks, :, place])
            wide = scale.repeat_interleave(SCALE_DIMS, -1)
            assert ((got - want).abs() <= wide * (0.5 + 2.0 ** -20) + 2 * off).all()
    for x in names:
        assert torch.equal(getattr(s, x).cpu().transpose(1, 2)[~touched].view(torch.uint8), before[x].cpu().transpose(1, 2)[~touched].view(torch.uint8)), x
    if with_q:
        assert (q_out[sum(s.new):] == 7.0).all()


@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", [
    (4, 2, 64, 128, [0], [1]), (16, 8, 128, 256, [63, 0, 255, 300], [1, 1, 1, 1]), (3, 1, 128, 128, [100, 5], [200, 0]),
    (10, 5, 64, 384, [383, 0], [2, 131]), (32, 8, 64, 128, [37], [700]), (16, 8, 128, 1024, [900], [400])])
@pytest.mark.parametrize("fused", [True, False])
def test_append(Hq, Hkv, d, block, old, new, fused):
    import paper_2603_02631_b200 as spf
    s = make_step4(Hq, Hkv, d, block, old, new, seed=d + Hq, behind=3, fused=fused)
    check(spf, s, rope_table(2000, d))


@pytest.mark.parametrize("rot_dim", [16, 32, 48, 64, 80, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_of_the_head_is_rotated(rot_dim, interleaved):
    import paper_2603_02631_b200 as spf
    d = 64 if rot_dim <= 64 else 128
    s = make_step4(4, 2, d, 128, [120, 7], [30, 9], seed=rot_dim)
    positions = torch.randint(0, 5000, (s.rows,), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    check(spf, s, rope_table(5000, rot_dim), positions, interleaved)


def test_without_rotation_and_without_queries():
    import paper_2603_02631_b200 as spf
    s = make_step4(4, 2, 128, 128, [120, 0], [30, 9], seed=2)
    check(spf, s)
    check(spf, make_step4(4, 2, 64, 128, [120, 0], [30, 9], seed=3), rope_table(200, 64), with_q=False)


def test_zeros_extremes_infinities_and_nan():
    import paper_2603_02631_b200 as spf
    s = make_step4(2, 1, 64, 128, [0], [6], seed=4)
    inf, nan = float("inf"), float("nan")
    s.v[0] = 0
    s.v[1, 0, :32], s.v[1, 0, 32:] = 3.3e38, -2.0 ** -130
    s.v[2, 0, 3], s.v[2, 0, 9] = inf, -inf
    s.v[3, 0, 40] = nan
    s.v[4, 0, :32] = inf
    append(spf, s)
    block = int(s.table[0, 0])
    scale, got = s.v_scale[block, 0, :6].cpu().double(), values(s.v_pool[block, 0, :6], s.v_scale[block, 0, :6])
    assert (got[0] == 0).all() and (scale[0] == 2.0 ** -100).all()
    assert ((got[1, :32] - s.v[1, 0, :32].double().cpu()).abs() <= scale[1, 0] * 0.5 * (1 + 2.0 ** -20)).all() and (got[1, 32:] == 0).all()
    finite = [i for i in range(32) if i not in (3, 9)]
    assert float(scale[2, 0]) == short_scale(float(s.v[2, 0, finite].abs().max()))
    assert got[2, 3] == 7 * scale[2, 0] and got[2, 9] == -7 * scale[2, 0]
    assert torch.isnan(got[3, 32:]).all() and torch.isfinite(got[3, :32]).all()
    assert (got[4, :32] == 7 * 2.0 ** -100).all()


def test_places_outside_are_reported_and_left_out():
    import paper_2603_02631_b200 as spf
    s = make_step4(2, 1, 64, 128, [120, 100], [20, 4], seed=5)
    bad = int(s.table[0, 1])
    s.table[0, 1] = s.k_pool.shape[0] + 5
    before = s.k_pool.clone()
    q = append(spf, s, status=-7)
    assert torch.equal(s.k_pool[bad], before[bad])
    assert (q[8:20] == 7).all() and not (q[20:] == 7).any()
    here = int(s.table[1, 0])
    assert not torch.equal(s.k_pool[here, :, 100:104], before[here, :, 100:104])


def test_any_order_of_steps_gives_the_same_bytes():
    """Tokens have scales of their own: one step of a prompt, and its tokens one by one, leave the same cache."""
    import paper_2603_02631_b200 as spf
    whole, single = (make_step4(2, 2, 128, 128, [0], [150], seed=6) for _ in range(2))
    append(spf, whole, rope_table(200, 128))
    k, v, q = single.k, single.v, single.q
    for t in range(150):
        single.row_start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        single.seq_lens = torch.tensor([t + 1], dtype=torch.int32, device="cuda")
        single.k, single.v, single.q, single.rows = k[t:t + 1], v[t:t + 1], q[t:t + 1], 1
        append(spf, single, rope_table(200, 128))
    for x in ("k_pool", "v_pool", "k_scale", "v_scale"):
        assert torch.equal(getattr(whole, x).view(torch.uint8), getattr(single, x).view(torch.uint8)), x
