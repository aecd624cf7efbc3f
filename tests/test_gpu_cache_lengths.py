"""Lengths at the ends of 32 bits: reported, and nothing is written for them; the sequence beside them is as it should be."""
import pytest
import torch

from attend_reference import check
from kv_reference import make_step

pytestmark = pytest.mark.gpu

LENGTHS = [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 63, 2 ** 31 - 64, 2 ** 31 - 128, 2 ** 30, -1, -2 ** 30, -2 ** 31 + 1, -2 ** 31]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("length", LENGTHS)
def test_append(length, new, bits):
    import paper_2603_02631_b200 as spf
    for with_q in (False, True):
        s = make_step(4, 2, 64, 128, [30, 100], [5, new], bits, seed=new)
        want = make_step(4, 2, 64, 128, [30, 100], [5, new], bits, seed=new)
        spf.spf_kv_append(want.cache(spf), spf.KvStep(want.row_start[:2].contiguous(), want.seq_lens[:1].contiguous(), want.table[:1].contiguous(), 5),
                          want.k, want.v)
        s.seq_lens[1] = length
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        q_out = torch.full_like(s.q, 7.0).contiguous()
        spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q if with_q else None, q_out if with_q else None, dev_status=status)
        torch.cuda.synchronize()
        assert int(status.item()) == -7
        for name in ("k_pool", "v_pool", "k_scale", "v_scale"):
            assert bits == 16 and "scale" in name or torch.equal(getattr(s, name).view(torch.uint8), getattr(want, name).view(torch.uint8)), name
        assert (q_out[5:] == 7.0).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("length", LENGTHS)
def test_attend(length, new, bits):
    """A negative length leaves the sequence's rows without keys; one beyond the table sees what the table has."""
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, 64, 128, [30, 100], [5, new], bits, seed=new)
    s.seq_lens[1] = length
    out, lse = torch.full_like(s.q, 7.0).contiguous(), torch.full((s.rows, 4), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), s.step(spf), s.q), dtype=torch.uint8, device="cuda")
    spf.spf_attend(s.cache(spf), s.step(spf), s.q, out, ws, lse, dev_status=status)
    torch.cuda.synchronize()
    assert int(status.item()) == -7
    if length < 0:
        assert (out[5:] == 0).all() and (lse[5:] == -float("inf")).all()
    s.new = [5, 0]
    check(s, out, lse)
