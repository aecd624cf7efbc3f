"""spf_kv_append against the 64-bit reference: rotated queries and keys, bf16 and 8-bit pools, everything else untouched."""
import pytest
import torch

from kv_reference import SCALE_TOKENS, e4m3_values, make_step, pow2_scale, rope_table, rotate

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8        # half a step, relative
E4M3 = 2.0 ** -4


def _check(spf, s, rope=None, positions=None, interleaved=False, with_q=True, in_place=False):
    before = {x: getattr(s, x).clone() for x in ("k_pool", "v_pool")}
    scales = {x: None if getattr(s, x) is None else getattr(s, x).clone() for x in ("k_scale", "v_scale")}
    q_in = s.q.clone()
    q_out = s.q if in_place else torch.full((s.rows, s.Hq, s.d), 7.0, dtype=torch.bfloat16, device=s.q.device)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    r = None if rope is None else spf.Rope(rope.cuda(), None if positions is None else positions.cuda(), interleaved)
    spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q if with_q else None, q_out if with_q else None, r, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    seen = {x: torch.zeros(before[x].shape[:3], dtype=torch.bool) for x in before}
    for b, (old, new) in enumerate(zip(s.old, s.new)):
        if new == 0:
            continue
        start = int(s.row_start[b])
        rows = slice(start, start + new)
        pos = torch.arange(old, old + new)
        at = pos if positions is None else positions[rows].long()
        for name, x, pool, scale in (("q", q_in, None, None), ("k", s.k, s.k_pool, s.k_scale), ("v", s.v, s.v_pool, s.v_scale)):
            if name == "q" and not with_q:
                continue
            x = x[rows]
            if rope is not None and name != "v":
                want, off = rotate(x, rope, at, interleaved)
            else:
                want, off = x.double().cpu(), torch.zeros(x.shape, dtype=torch.float64)
            if name == "q":
                got = q_out[rows].double().cpu()
                assert ((got - want).abs() <= BF16 * want.abs() + 2 * off).all()
                continue
            blocks, place = s.table.cpu()[b][pos // s.block].long(), pos % s.block
            seen[name + "_pool"][blocks, :, place] = True
            if scale is None:
                got = pool.cpu()[blocks, :, place].double()
                assert ((got - want).abs() <= BF16 * want.abs() + 2 * off).all()
                continue
            sc = scale.cpu()[blocks, :, place // SCALE_TOKENS].double()
            got = e4m3_values(pool.cpu()[blocks, :, place]) * sc[..., None]
            # half a step of the format (2^-10 of the scale where it is subnormal)
            assert ((got - want).abs() <= torch.maximum(E4M3 * want.abs(), 2.0 ** -10 * sc[..., None]) + 2 * off).all()
            for g in range(old // SCALE_TOKENS, (old + new - 1) // SCALE_TOKENS + 1):
                lo, hi = max(g * SCALE_TOKENS, old), min((g + 1) * SCALE_TOKENS, old + new)
                block, cell = int(s.table[b, lo // s.block]), (g * SCALE_TOKENS % s.block) // SCALE_TOKENS
                for h in range(s.Hkv):
                    need = pow2_scale(float(want[lo - old:hi - old, h].abs().max()))
                    held = float(scales[name + "_scale"][block, h, cell]) if lo > g * SCALE_TOKENS else 0.0
                    assert float(scale[block, h, cell]) == max(need, held)
                    if lo > g * SCALE_TOKENS:            # tokens from before the step: rounded once more, to the new scale
                        first = g * SCALE_TOKENS % s.block
                        part = slice(first, first + lo - g * SCALE_TOKENS)
                        was = e4m3_values(before[name + "_pool"][block, h, part].cpu()) * held
                        now = e4m3_values(pool[block, h, part].cpu()) * max(need, held)
                        assert ((now - was).abs() <= 2.0 ** -10 * max(need, held)).all()
                        if held >= need:
                            assert torch.equal(now, was)
                        seen[name + "_pool"][block, h, part] = True
    for name in before:                                   # nothing else in the pools has changed
        same = getattr(s, name).cpu().view(torch.uint8) == before[name].cpu().view(torch.uint8)
        assert same.view(*seen[name].shape, -1).all(-1)[~seen[name]].all()
    if with_q and not in_place:
        assert (q_out[sum(s.new):] == 7.0).all()          # rows behind the last sequence


CASES = [
    # Hq, Hkv, d, block, tokens before, new tokens
    (4, 2, 64, 128, [0], [1]),                              # the first token of a cache
    (4, 2, 64, 128, [127], [2]),                            # over a block's end
    (16, 8, 128, 256, [255, 0, 64, 63, 130], [1, 1, 1, 1, 1]),
    (6, 2, 64, 384, [5, 300, 0, 77], [200, 0, 1, 131]),     # a block of three tiles, a sequence without new tokens
    (3, 1, 128, 128, [31], [700]),
    (8, 8, 64, 1024, [1000, 2000], [100, 65]),
    (32, 8, 64, 4096, [0, 10], [1500, 2100]),               # enough rows for several heads a thread
]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", CASES)
def test_append_with_rotation(Hq, Hkv, d, block, old, new, bits):
    import paper_2603_02631_b200 as spf
    s = make_step(Hq, Hkv, d, block, old, new, bits, seed=d + block, behind=3)
    _check(spf, s, rope_table(max(a + b for a, b in zip(old, new)), d))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rot_dim,interleaved", [(16, False), (32, True), (64, True), (64, False)])
def test_partial_and_interleaved_rotation_with_given_positions(rot_dim, interleaved, bits):
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, 64, 128, [40, 90], [30, 60], bits, seed=rot_dim, behind=2, fused=False)
    positions = torch.randint(0, 5000, (s.rows,), generator=torch.Generator().manual_seed(1)).to(torch.int32)
    _check(spf, s, rope_table(5000, rot_dim), positions, interleaved)


@pytest.mark.parametrize("bits", [16, 8])
def test_without_rotation_without_queries_and_in_place(bits):
    import paper_2603_02631_b200 as spf
    _check(spf, make_step(4, 2, 128, 128, [3, 200], [9, 61], bits, seed=1))
    _check(spf, make_step(4, 2, 128, 128, [3, 200], [9, 61], bits, seed=2), rope_table(300, 128), with_q=False)
    _check(spf, make_step(4, 2, 128, 128, [3, 200], [9, 61], bits, seed=3), rope_table(300, 128), in_place=True)


def test_a_group_of_tokens_grows_its_scale():
    """Tokens that come one by one, each louder than the one before: the group's earlier bytes follow the scale."""
    import paper_2603_02631_b200 as spf
    s = make_step(2, 1, 64, 128, [0], [1], 8, seed=5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(9)
    written = []
    for t in range(70):
        x = (torch.randn((1, 1, 64), generator=gen) * 1.3 ** t).to(torch.bfloat16).cuda()
        step = spf.KvStep(s.row_start, torch.tensor([t + 1], dtype=torch.int32, device="cuda"), s.table, 1)
        spf.spf_kv_append(s.cache(spf), step, x, x, dev_status=status)
        written.append(x[0, 0].double().cpu())
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    block = int(s.table[0, 0])
    for pool, scale in ((s.k_pool, s.k_scale), (s.v_pool, s.v_scale)):
        for g, (lo, hi) in enumerate(((0, 64), (64, 70))):
            sc = float(scale[block, 0, g])
            assert sc == pow2_scale(max(float(w.abs().max()) for w in written[lo:hi]))
            got = e4m3_values(pool[block, 0, lo:hi].cpu()) * sc
            want = torch.stack(written[lo:hi])
            # a value is rounded when it comes (half a step) and at each growth that leaves it subnormal: the growths' half
            # steps are 2^-10 of scales that double, so they add up to less than 2^-9 of the last one
            assert ((got - want).abs() <= E4M3 * want.abs() + 2.0 ** -9 * sc).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_values_that_are_not_finite_and_zeros(bits):
    import paper_2603_02631_b200 as spf
    s = make_step(1, 1, 64, 128, [0], [3], bits, seed=6)
    s.k[0], s.v[0] = 0.0, 0.0
    s.v[1, 0, 5], s.v[1, 0, 6], s.v[2, 0, 7] = float("inf"), float("-inf"), float("nan")
    spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v)
    torch.cuda.synchronize()
    block = int(s.table[0, 0])
    if bits == 16:
        assert torch.equal(s.v_pool[block, 0, :3].view(torch.int16), s.v[:, 0].contiguous().view(torch.int16))
        return
    scale, got = float(s.v_scale[block, 0, 0]), e4m3_values(s.v_pool[block, 0, :3].cpu())
    rest = s.v[:, 0].double().cpu()
    rest[~torch.isfinite(rest)] = 0
    assert scale == pow2_scale(float(rest.abs().max()))
    assert got[1, 5] == 448 and got[1, 6] == -448 and torch.isnan(got[2, 7]) and int(torch.isnan(got).sum()) == 1
    assert (got[0] == 0).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_rows_outside_the_cache_are_left_out_and_reported(bits):
    import paper_2603_02631_b200 as spf
    # rows of the step that have no place in each case; rows 0 to 4 are the first sequence's, 5 to 64 the second's, which lie at
    # 100 ... 159, at 228 ... 287 ("length": its table ends at 256) or at -40 ... 19 ("negative")
    cases = {"block": range(33, 65), "length": range(33, 65), "position": [20], "negative": range(5, 45)}
    for what, left_out in cases.items():
        s = make_step(2, 1, 64, 128, [10, 100], [5, 60], bits, seed=8)
        clean = {x: getattr(s, x).clone() for x in ("k_pool", "v_pool")}
        rope, positions = rope_table(200, 64), torch.arange(65, dtype=torch.int32)
        if what == "block":
            s.table[1, 1] = s.k_pool.shape[0]             # the second sequence's tokens from 128 on have no block
        elif what == "length":
            s.seq_lens[1] += 128                          # behind its table: tokens from 256 on
        elif what == "position":
            positions[20] = 200
        else:
            s.seq_lens[1] = 20                            # fewer tokens than new ones
        q_out = torch.full((s.rows, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q, q_out, spf.Rope(rope.cuda(), positions.cuda()), status)
        torch.cuda.synchronize()
        assert int(status.item()) == -7, what
        first = int(s.table[0, 0])
        assert not torch.equal(clean["k_pool"][first, 0, 10:15], s.k_pool[first, 0, 10:15])    # the first sequence is written
        done = [r for r in range(65) if r not in left_out]
        assert (q_out[list(left_out)] == 7.0).all() and not (q_out[done] == 7.0).all((1, 2)).any(), what


@pytest.mark.parametrize("bits", [16, 8])
def test_many_sequences_and_a_graph_that_is_replayed_with_other_lengths(bits):
    import paper_2603_02631_b200 as spf
    old, new = [(7 * b) % 300 for b in range(300)], [1] * 300
    s = make_step(2, 1, 64, 128, old, new, bits, seed=11)
    rope = rope_table(400, 64)
    pools = s.k_pool.clone(), s.v_pool.clone()
    scales = None if bits == 16 else (s.k_scale.clone(), s.v_scale.clone())
    r = spf.Rope(rope.cuda())
    q_out = torch.empty_like(s.q)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q, q_out, r, status)
    s.seq_lens += 5                                        # other lengths, the same graph (and the history is what it was)
    s.old = [x + 5 for x in old]
    s.table.copy_(torch.arange(s.table.numel(), dtype=torch.int32).view(s.table.shape) % s.k_pool.shape[0])
    graph.replay()
    torch.cuda.synchronize()
    by_graph = s.k_pool.clone(), s.v_pool.clone(), q_out.clone()
    s.k_pool.copy_(pools[0]), s.v_pool.copy_(pools[1])
    if scales:
        s.k_scale.copy_(scales[0]), s.v_scale.copy_(scales[1])
    spf.spf_kv_append(s.cache(spf), s.step(spf), s.k, s.v, s.q, q_out, r, status)
    torch.cuda.synchronize()
    # blocks that two sequences of this table share are written by both; those of one sequence alone are compared
    ids, count = s.table.flatten().unique(return_counts=True)
    alone = ids[count == 1].long()
    assert torch.equal(by_graph[0][alone], s.k_pool[alone]) and torch.equal(by_graph[1][alone], s.v_pool[alone])
    assert torch.equal(by_graph[2], q_out)


@pytest.mark.parametrize("Hkv,rot_dim", [(3, 64), (8, 32), (12, 64)])
def test_several_heads_of_a_group_to_a_cta(Hkv, rot_dim):
    """Enough 8-bit groups that a CTA makes several heads' keys and values of one, a number that does not divide the heads among them."""
    import paper_2603_02631_b200 as spf
    s = make_step(2 * Hkv, Hkv, 64, 128, [70, 0], [4500, 5000], 8, seed=Hkv)
    _check(spf, s, rope_table(6000, rot_dim))
