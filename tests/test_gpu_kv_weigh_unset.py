"""spf_kv_weigh on a ledger whose memory was never written: a decay of 0 replaces what is held."""
import pytest
import torch

from ledger_reference import any_step, ledger_of
from test_gpu_kv_weigh import reference_lse, weigh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new", [1, 9, 150])
def test_a_decay_of_zero_does_not_look_at_what_is_held(bits, new):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, 4, 2, 64, 128, [300], [new], 8)
    lse = reference_lse(s, bits)
    clean, unset = torch.zeros_like(ledger_of(s, 5)[0]), torch.zeros_like(ledger_of(s, 5)[0])
    unset[..., 0::3], unset[..., 1::3], unset[..., 2::3] = float("nan"), float("inf"), -float("inf")
    weigh(spf, s, lse, clean, None, decay=0.0)
    weigh(spf, s, lse, unset, None, decay=0.0)
    key = torch.arange(300 + new)
    at, place = s.table.cpu()[0][key // 128].long(), key % 128
    assert torch.equal(unset.cpu()[at, :, place], clean.cpu()[at, :, place])
