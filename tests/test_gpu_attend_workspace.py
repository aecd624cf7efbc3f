"""Workspaces of spf_attend: what is refused, and that one of a step with more new tokens serves every smaller step."""
import pytest
import torch

from attend_reference import check, gpu_step
from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_new", [0, -1, 1 << 31, (1 << 32) + 1, -(1 << 40) + 5])
def test_hints_that_are_no_number_of_tokens_are_refused(max_new):
    """Also those whose low 32 bits are one."""
    import paper_2603_02631_b200 as spf
    s = gpu_step(4, 2, 64, 128, [100], [1], 16)
    step = spf.KvStep(s.row_start, s.seq_lens, s.table, max_new)
    with pytest.raises(ValueError):
        spf.spf_attend_workspace_bytes(s.cache(spf), step, s.q)
    with pytest.raises(ValueError):
        spf.spf_attend(s.cache(spf), step, s.q, torch.empty_like(s.q), torch.empty(1 << 26, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d", [(8, 8, 64), (8, 2, 128), (16, 2, 64)])
def test_a_workspace_serves_steps_of_fewer_tokens(Hq, Hkv, d, bits):
    import paper_2603_02631_b200 as spf
    largest = gpu_step(Hq, Hkv, d, 128, [100], [600], bits)
    ws = torch.empty(spf.spf_attend_workspace_bytes(largest.cache(spf), largest.step(spf), largest.q) + 256, dtype=torch.uint8, device="cuda")
    for new in (600, 40, 9, 8, 5, 4, 3, 2, 1):
        s = gpu_step(Hq, Hkv, d, 128, [3000, 5], [new, 1], bits, seed=new)
        assert spf.spf_attend_workspace_bytes(s.cache(spf), s.step(spf), s.q) <= ws.numel() - 256
        ws.fill_(255)
        check(s, *run(spf, s, workspace=ws[:-256]))
        assert (ws[-256:] == 255).all()                     # nothing is written behind it
