"""A draft model's steps on a cache that is cut to a budget, as they follow one another: append, attend, weigh, evict, and on over what is left;
eager and replayed, on 4-bit, 8-bit and bf16 caches.  After a cut each head's cache holds its own tokens, so the reference follows heads."""
import math

import pytest
import torch

from kv4_reference import SCALE_DIMS
from kv_reference import SCALE_TOKENS, e4m3_values, rope_table
from kv4_reference import values as values4

pytestmark = pytest.mark.gpu

Hq, Hkv, D, BLOCK, KEEP, FIRST, RECENT = 8, 2, 64, 128, 200, 4, 32


class Draft:
    """Two sequences, blocks for them and for what is copied, everything on the GPU."""

    def __init__(self, spf, bits, seed):
        gen = torch.Generator().manual_seed(seed)
        self.spf, self.bits, self.gen = spf, bits, gen
        blocks = 24
        shape = (blocks, Hkv, BLOCK, D if bits != 4 else D // 2)
        kind = torch.bfloat16 if bits == 16 else torch.uint8
        make = lambda: torch.zeros(shape, dtype=kind, device="cuda")  # noqa: E731
        scale = lambda: (None if bits == 16 else torch.ones((blocks, Hkv, BLOCK // SCALE_TOKENS), device="cuda") if bits == 8 else  # noqa: E731
                         torch.ones((blocks, Hkv, BLOCK, D // SCALE_DIMS), dtype=torch.bfloat16, device="cuda"))
        self.cache = spf.KvCache(make(), make(), scale(), scale())
        self.ledger = spf.KvLedger(torch.zeros((blocks, Hkv, BLOCK), device="cuda"), torch.zeros((blocks, Hkv, BLOCK), dtype=torch.int32, device="cuda"))
        order = torch.randperm(blocks, generator=gen).to(torch.int32)
        self.tables = [order[0:8].view(2, 4).contiguous().cuda(), order[8:16].view(2, 4).contiguous().cuda()]
        self.lens = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.n_seen = torch.zeros(2, dtype=torch.int32, device="cuda")
        self.keep = torch.full((2,), KEEP, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.rope = spf.Rope(rope_table(4000, D).cuda())
        self.evict_ws = torch.empty(spf.spf_kv_evict_workspace_bytes(self.cache, self.tables[0]), dtype=torch.uint8, device="cuda")

    def inputs(self, new):
        rows = sum(new)
        qkv = torch.randn((rows, Hq + 2 * Hkv, D), generator=self.gen).to(torch.bfloat16).cuda()
        starts = torch.tensor([0, new[0], rows], dtype=torch.int32, device="cuda")
        return qkv, starts

    def step(self, qkv, starts, positions, table, max_new):
        """One step; lens hold the new tokens already."""
        spf = self.spf
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        step = spf.KvStep(starts, self.lens, table, max_new)
        q_rot, out = torch.zeros_like(q).contiguous(), torch.zeros_like(q).contiguous()
        lse = torch.zeros((len(q), Hq), device="cuda")
        ws = torch.empty(spf.spf_attend_workspace_bytes(self.cache, step, q), dtype=torch.uint8, device="cuda")
        rope = spf.Rope(self.rope.table, positions)
        spf.spf_kv_append(self.cache, step, k, v, q, q_rot, rope, self.status)
        spf.spf_attend(self.cache, step, q_rot, out, ws, lse, dev_status=self.status)
        spf.spf_kv_weigh(self.cache, step, q_rot, lse, self.ledger, positions=positions, decay=0.9, dev_status=self.status)
        return q_rot, out, lse

    def cut(self, table, to):
        self.spf.spf_kv_evict(self.cache, self.ledger, self.lens, table, self.keep, to, self.lens, self.evict_ws, FIRST, RECENT, self.n_seen, self.status)

    def held(self, table, b, h):
        """(keys, values, weights, positions) that a sequence's head has, float64."""
        n = int(self.lens[b])
        ids = table[b].long().cpu()
        c = self.cache
        out = []
        for pool, scale in ((c.k_pool, c.k_scale), (c.v_pool, c.v_scale)):
            x = pool.cpu()[ids, h]
            if self.bits == 16:
                x = x.double()
            elif self.bits == 8:
                x = e4m3_values(x) * scale.cpu()[ids, h].double().repeat_interleave(SCALE_TOKENS, -1)[..., None]
            else:
                x = values4(x, scale.cpu()[ids, h])
            out.append(x.flatten(0, 1)[:n])
        return (*out, self.ledger.weight.cpu()[ids, h].flatten()[:n].double(), self.ledger.position.cpu()[ids, h].flatten()[:n])


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_prompt_then_tokens_on_a_bounded_cache(bits):
    import paper_2603_02631_b200 as spf
    d = Draft(spf, bits, 3)
    current, spare = d.tables
    for new in ([300, 130], [90, 64], [1, 1], [1, 0], [1, 1], [3, 2]):
        qkv, starts = d.inputs(new)
        before = [[d.held(current, b, h) for h in range(Hkv)] for b in range(2)]
        d.lens += torch.tensor(new, dtype=torch.int32, device="cuda")
        d.n_seen += torch.tensor(new, dtype=torch.int32, device="cuda")
        positions = torch.cat([torch.arange(int(s) - n, int(s), dtype=torch.int32) for s, n in zip(d.n_seen.tolist(), new)]).cuda()
        q, out, lse = d.step(qkv, starts, positions, current, max(new))
        torch.cuda.synchronize()
        assert int(d.status) == 0
        for b in range(2):
            rows = slice(int(starts[b]), int(starts[b + 1]))
            for h in range(Hkv):
                k, v, weight, position = d.held(current, b, h)
                old = len(before[b][h][2])
                assert torch.equal(position[:old], before[b][h][3]) and torch.equal(position[old:], positions[rows].cpu())
                got = torch.zeros(len(k), dtype=torch.float64)
                for g in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                    z = q[rows, g].double().cpu() @ k.T / math.sqrt(D)
                    hidden = torch.arange(len(k))[None, :] > old + torch.arange(new[b])[:, None]
                    z = z.masked_fill(hidden, -math.inf)
                    p = torch.softmax(z, -1)
                    want = p @ v
                    # half a step of bf16 of the output and of the weights; logits' rounding is far below these
                    assert ((out[rows, g].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -7 + 2.0 ** -10) * (p @ v.abs()) + 2.0 ** -13).all()
                    own = torch.exp(z - lse[rows, g].double().cpu()[:, None]).masked_fill(hidden, 0.0)
                    got += own.sum(0)
                want = torch.cat([before[b][h][2] * 0.9, torch.zeros(new[b], dtype=torch.float64)]) + got
                if new[b] == 0:
                    want = before[b][h][2]
                assert ((weight - want).abs() <= 2.0 ** -13 * want + 2.0 ** -30).all()
        if max(d.lens.tolist()) > KEEP + 2:
            held = [[d.held(current, b, h) for h in range(Hkv)] for b in range(2)]
            d.cut(current, spare)
            current, spare = spare, current
            torch.cuda.synchronize()
            assert int(d.status) == 0 and max(d.lens.tolist()) <= KEEP
            for b in range(2):
                for h in range(Hkv):
                    k, v, weight, position = d.held(current, b, h)
                    was = {int(p): i for i, p in enumerate(held[b][h][3])}
                    at = torch.tensor([was[int(p)] for p in position])
                    assert (at[1:] > at[:-1]).all()                          # in the order of the places
                    assert torch.equal(weight, held[b][h][2][at])
                    gone = torch.ones(len(held[b][h][2]), dtype=torch.bool)
                    gone[at] = False
                    protected = (position < FIRST) | (position >= int(d.n_seen[b]) - RECENT)
                    if gone.any() and (~protected).any():
                        assert held[b][h][2][gone].max() <= weight[~protected].min()
                    slack = 0 if bits != 8 else 2.0 ** -4 * v.abs() + 2.0 ** -9 * v.abs().max()
                    assert ((v - held[b][h][1][at]).abs() <= slack).all()


@pytest.mark.parametrize("bits", [4, 8, 16])
def test_a_captured_step_and_cut_replayed_against_eager_ones(bits):
    import paper_2603_02631_b200 as spf

    def prepared():
        d = Draft(spf, bits, 5)
        qkv, starts = d.inputs([190, 150])
        d.lens += torch.tensor([190, 150], dtype=torch.int32, device="cuda")
        d.n_seen.copy_(d.lens)
        d.step(qkv, starts, torch.cat([torch.arange(190), torch.arange(150)]).to(torch.int32).cuda(), d.tables[0], 190)
        return d

    eager, replayed = prepared(), prepared()
    one = torch.ones(2, dtype=torch.int32, device="cuda")
    qkv, starts = torch.zeros((2, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    other = {}

    def turn(d, key, positions):
        # one token a sequence, then a cut to the other blocks and back again: both tables are in the graph
        q, out, lse = d.step(qkv, starts, positions, d.tables[0], 1)
        d.cut(d.tables[0], d.tables[1])
        d.cut(d.tables[1], d.tables[0])
        other[key] = (out, lse)

    positions = torch.zeros(2, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        turn(replayed, "replayed", positions)
    gen = torch.Generator().manual_seed(9)
    for _ in range(25):
        qkv.copy_(torch.randn(qkv.shape, generator=gen).to(torch.bfloat16))
        for d in (eager, replayed):
            d.lens += one
            d.n_seen += one
        positions.copy_(eager.n_seen - 1)
        turn(eager, "eager", positions)
        graph.replay()
        torch.cuda.synchronize()
        assert int(eager.status) == 0 and int(replayed.status) == 0
        assert torch.equal(eager.lens, replayed.lens) and int(eager.lens[0]) <= KEEP
        for a, b in zip(other["eager"], other["replayed"]):
            assert torch.equal(a, b)
        assert torch.equal(eager.ledger.weight, replayed.ledger.weight) and torch.equal(eager.ledger.position, replayed.ledger.position)
        assert torch.equal(eager.cache.k_pool.view(torch.uint8), replayed.cache.k_pool.view(torch.uint8))


def test_calls_on_another_stream_and_two_at_once():
    import paper_2603_02631_b200 as spf
    drafts = [Draft(spf, 4, s) for s in (7, 8)]
    want = []
    for d in drafts:
        qkv, starts = d.inputs([230, 210])
        d.lens += torch.tensor([230, 210], dtype=torch.int32, device="cuda")
        d.n_seen.copy_(d.lens)
        positions = torch.cat([torch.arange(230), torch.arange(210)]).to(torch.int32).cuda()
        d.step(qkv, starts, positions, d.tables[0], 230)
        d.cut(d.tables[0], d.tables[1])
        want.append((d.ledger.weight.clone(), d.cache.k_pool.clone(), d.lens.clone()))
    streams = [torch.cuda.Stream() for _ in drafts]
    again = [Draft(spf, 4, s) for s in (7, 8)]
    ready = []
    for d in again:
        qkv, starts = d.inputs([230, 210])
        d.lens += torch.tensor([230, 210], dtype=torch.int32, device="cuda")
        d.n_seen.copy_(d.lens)
        ready.append((qkv, starts, torch.cat([torch.arange(230), torch.arange(210)]).to(torch.int32).cuda()))
    torch.cuda.synchronize()
    for d, s, (qkv, starts, positions) in zip(again, streams, ready):
        with torch.cuda.stream(s):
            d.step(qkv, starts, positions, d.tables[0], 230)
            d.cut(d.tables[0], d.tables[1])
    torch.cuda.synchronize()
    for d, (weight, pool, lens) in zip(again, want):
        assert torch.equal(d.ledger.weight, weight) and torch.equal(d.cache.k_pool, pool) and torch.equal(d.lens, lens)
