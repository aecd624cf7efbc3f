"""A chunk's append and attention captured once and replayed with other lengths, sequences that gain or lose tokens, and empty ones."""
import pytest
import torch

from attend_reference import check, gpu_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_a_chunk_replayed_with_other_splits(d, bits):
    import paper_2603_02631_b200 as spf
    s = gpu_step(8, 2, d, 128, [3000, 2000, 2500], [300, 300, 300], bits, seed=d + bits)
    old, first = list(s.old), torch.zeros(3, dtype=torch.int32, device="cuda")
    step, cache = s.step(spf, 900), s.cache(spf)
    ws = torch.empty(spf.spf_attend_workspace_bytes(cache, step, s.q), dtype=torch.uint8, device="cuda")
    out, lse, status = torch.zeros_like(s.q), torch.zeros((900, 8), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        spf.spf_attend(cache, step, s.q, out, ws, lse, first, dev_status=status)
    for new, begin in (([300, 300, 300], [0, 0, 0]), ([1, 0, 299], [100, 5, 2600]), ([0, 0, 0], [0, 0, 0]), ([290, 250, 200], [3200, 2249, 0]), ([0, 300, 0], [0, 64, 0])):
        starts = [sum(new[:b]) for b in range(4)]
        s.row_start.copy_(torch.tensor(starts, dtype=torch.int32))
        s.seq_lens.copy_(torch.tensor([a + c for a, c in zip(old, new)], dtype=torch.int32))
        first.copy_(torch.tensor(begin, dtype=torch.int32))
        out.fill_(7.0), lse.fill_(7.0), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        assert (out[sum(new):] == 7.0).all() and (lse[sum(new):] == 7.0).all()
        s.new, s.old = new, old
        check(s, out, lse, first=begin)
