"""spf_kv_append with enough rows for the variants of many heads a thread and a CTA, at both head dimensions."""
import pytest
import torch

from kv_reference import make_step, rope_table
from test_gpu_kv_append import _check

pytestmark = pytest.mark.gpu


def enough(s):
    return sum(s.new) * (s.Hq + 2 * s.Hkv) * (s.d // 16) > 148 * 2048


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,rot_dim,interleaved,given", [
    (6, 3, 128, 128, False, False), (7, 7, 128, 32, True, True), (24, 12, 128, 128, True, False), (5, 5, 64, 32, False, True), (9, 3, 64, 64, True, True),
    (1, 1, 128, 96, False, True),
])
def test_many_rows(Hq, Hkv, d, rot_dim, interleaved, given, bits):
    import paper_2603_02631_b200 as spf
    few = 148 * 2048 // ((Hq + 2 * Hkv) * d // 16) // 2
    s = make_step(Hq, Hkv, d, 384, [70, 0, 1000, 5], [few + 77, few, 0, 63], bits, seed=Hq + d, behind=3)
    assert enough(s)
    positions = torch.randint(0, 9000, (s.rows,), generator=torch.Generator().manual_seed(2)).to(torch.int32) if given else None
    _check(spf, s, rope_table(max(9000, 2 * few + 200), rot_dim), positions, interleaved)


@pytest.mark.parametrize("bits", [16, 8])
def test_many_rows_without_rotation_without_queries_and_in_place(bits):
    import paper_2603_02631_b200 as spf
    shape = (8, 4, 128, 256, [100, 0], [2000, 900])
    s = make_step(*shape, bits, seed=1, fused=False)
    assert enough(s)
    _check(spf, s)
    _check(spf, make_step(*shape, bits, seed=2), rope_table(2100, 64), with_q=False)
    _check(spf, make_step(*shape, bits, seed=3), rope_table(2100, 128), in_place=True)
