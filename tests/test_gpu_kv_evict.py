"""spf_kv_evict against a plain sort: what is kept, where it goes, ties, NaN, budgets, every cache format."""
import random

import pytest
import torch

from kv_reference import SCALE_TOKENS, e4m3_values
from ledger_reference import any_step, kept_places, ledger_of, values_of

pytestmark = pytest.mark.gpu


def more_blocks(s, extra):
    """The step's pools with `extra` blocks more (of other bytes), in random order of all; returns the blocks that are new."""
    n = s.k_pool.shape[0]
    for x in ("k_pool", "v_pool", "k_scale", "v_scale"):
        t = getattr(s, x)
        if t is not None:
            setattr(s, x, torch.cat([t, t[torch.arange(extra) % n].flip(0)]).contiguous())
    return torch.arange(n, n + extra, dtype=torch.int32)[torch.randperm(extra, generator=torch.Generator().manual_seed(1))]


def cut(spf, s, weight, position, keep, to_table, n_first=0, n_recent=0, n_seen=None, status=0, in_place=False):
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    seen = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = s.seq_lens if in_place else torch.full_like(s.seq_lens, -9)
    ws = torch.full((spf.spf_kv_evict_workspace_bytes(s.cache(spf), to_table),), 255, dtype=torch.uint8, device="cuda")
    spf.spf_kv_evict(s.cache(spf), spf.KvLedger(weight, position), s.seq_lens, s.table, i32(keep), to_table, lens, ws, n_first, n_recent,
                     None if n_seen is None else i32(n_seen), seen)
    torch.cuda.synchronize()
    assert int(seen.item()) == status
    return lens


def check(spf, s, bits, keep, to_blocks, weight, position, n_first=0, n_recent=0, n_seen=None, in_place=False):
    names = ["k_pool", "v_pool"] + (["k_scale", "v_scale"] if bits != 16 else [])
    seqs = len(s.old)
    to_table = more_blocks(s, seqs * to_blocks).view(seqs, to_blocks).contiguous().cuda()
    blocks = s.k_pool.shape[0]
    weight = torch.cat([weight, torch.full((blocks - weight.shape[0], *weight.shape[1:]), -5.0, device="cuda")])
    if position is not None:
        position = torch.cat([position, torch.full((blocks - position.shape[0], *position.shape[1:]), -5, dtype=torch.int32, device="cuda")])
    before = {x: getattr(s, x).clone().cpu() for x in names} | {"weight": weight.clone().cpu()} | ({} if position is None else {"position": position.clone().cpu()})
    old_lens = s.seq_lens.tolist()
    lens = cut(spf, s, weight, position, keep, to_table, n_first, n_recent, n_seen, in_place=in_place)
    after = {x: getattr(s, x).cpu() for x in names} | {"weight": weight.cpu()} | ({} if position is None else {"position": position.cpu()})
    room, table, to = to_blocks * s.block, s.table.cpu().long(), to_table.cpu().long()
    left = [max(min(n, k, room), 0) for n, k in zip(old_lens, keep)]
    assert lens.tolist() == left
    want = {x: before[x].clone() for x in before}
    for b, n in enumerate(old_lens):
        place = torch.arange(n)
        at, off = table[b][place // s.block], place % s.block
        for h in range(s.Hkv):
            w = before["weight"][at, h, off]
            p = place if position is None else before["position"][at, h, off]
            kept = torch.tensor(kept_places(w.tolist(), p.tolist(), left[b], n_first, n_recent, n if n_seen is None else n_seen[b]), dtype=torch.long)
            src, dst = (at[kept], h, off[kept]), (to[b][torch.arange(left[b]) // s.block], h, torch.arange(left[b]) % s.block)
            for x in want:
                if bits != 8 or x in ("weight", "position"):
                    want[x][dst] = before[x][src]
            if bits == 8:
                for x in "kv":
                    scale = before[x + "_scale"][src[0], h, src[2] // SCALE_TOKENS]
                    for g in range(0, left[b], SCALE_TOKENS):
                        part = slice(g, g + SCALE_TOKENS)
                        top = scale[part].max()
                        want[x + "_scale"][dst[0][g], h, dst[2][g] // SCALE_TOKENS] = top
                        bytes_ = e4m3_values(before[x + "_pool"][src[0][part], h, src[2][part]]).float() * (scale[part] / top)[:, None]
                        want[x + "_pool"][dst[0][part], h, dst[2][part]] = bytes_.to(torch.float8_e4m3fn).view(torch.uint8)
    for x in want:
        a, b = (t.view(torch.int32) if t.dtype == torch.float32 else t.view(torch.int16) if t.dtype == torch.bfloat16 else t for t in (after[x], want[x]))
        assert torch.equal(a, b), x


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("Hkv,d,block,lens,keep", [
    (2, 64, 128, [300], [100]), (8, 128, 128, [63, 64, 65, 200], [64, 64, 64, 64]), (1, 128, 256, [1000, 0, 7], [513, 10, 7]),
    (3, 64, 384, [700, 129], [0, -4]), (2, 64, 128, [500, 500], [1, 499]), (1, 64, 128, [384, 300], [1000, 300])])
def test_cut(Hkv, d, block, lens, keep, bits):
    import paper_2603_02631_b200 as spf
    s = any_step(bits, Hkv, Hkv, d, block, lens, [0] * len(lens), d + block)
    weight, position = ledger_of(s, 1)
    check(spf, s, bits, keep, 4, weight, position)
    s = any_step(bits, Hkv, Hkv, d, block, lens, [0] * len(lens), d + block)
    check(spf, s, bits, keep, 4, ledger_of(s, 1)[0], None, n_first=3, n_recent=20, in_place=True)


def test_first_and_recent_ones_by_position():
    import paper_2603_02631_b200 as spf
    s = any_step(4, 2, 2, 64, 128, [300, 250], [0, 0], 3)
    weight, position = ledger_of(s, 1)
    position.copy_(torch.randint(0, 1000, position.shape, generator=torch.Generator().manual_seed(2)).to(torch.int32))
    check(spf, s, 4, [100, 200], 2, weight, position, n_first=50, n_recent=70, n_seen=[1000, 900])
    # more of them than are kept: those of the lowest places
    s = any_step(4, 2, 2, 64, 128, [300, 250], [0, 0], 3)
    check(spf, s, 4, [40, 5], 2, weight, position, n_first=500, n_recent=100, n_seen=[1000, 1000])


@pytest.mark.parametrize("parts", [1, 8])
def test_ties_zeros_infinities_and_nan(parts):
    import paper_2603_02631_b200 as spf
    gen = torch.Generator().manual_seed(4)
    for case in range(6):
        s = any_step(4, 1, 1, 64, 128, [700], [0], case)
        if parts == 8:                                     # a table with room for more tokens is ranked by more CTAs
            s.table = torch.cat([s.table, torch.full((1, 300), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
        weight, _ = ledger_of(s, 1)
        if case == 0:
            weight.fill_(0.25)
        elif case == 1:
            weight.copy_(torch.randint(0, 3, weight.shape, generator=gen).float())
        elif case == 2:
            weight.copy_(torch.where(torch.rand(weight.shape, generator=gen) < 0.5, 0.0, -0.0))
        elif case == 3:
            choice = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e-45, -1.0, 3.4e38])
            weight.copy_(choice[torch.randint(0, 6, weight.shape, generator=gen)])
        elif case == 4:
            weight.fill_(float("nan"))
        else:
            weight.copy_((torch.arange(weight.numel()) % 7).view(weight.shape).float() * 2.0 ** -140)
        check(spf, s, 4, [333], 4, weight, None, n_first=2, n_recent=9)


@pytest.mark.parametrize("block,n,keep,stride", [(4096, 30000, 9000, 0), (4096, 120001, 32768, 0), (4096, 300017, 777, 0), (128, 5000, 2048, 60)])
def test_long_sequences(block, n, keep, stride):
    """Several CTAs rank a sequence; the third has more numbers than they hold."""
    import paper_2603_02631_b200 as spf
    blocks = -(-n // block)
    to = -(-keep // block)
    pool = torch.randint(0, 256, (blocks + to, 1, block, 32), dtype=torch.uint8, device="cuda")
    scale = torch.ones((blocks + to, 1, block, 2), dtype=torch.bfloat16, device="cuda")
    cache = spf.KvCache(pool, pool.clone(), scale, scale.clone())
    perm = torch.randperm(blocks + to, device="cuda").to(torch.int32)
    table, to_table = torch.full((1, blocks + stride), -1, dtype=torch.int32, device="cuda"), perm[blocks:].view(1, to).contiguous()
    table[0, :blocks] = perm[:blocks]
    weight = torch.randint(0, 5000, (blocks + to, 1, block), device="cuda").float()        # with ties
    position = torch.zeros((blocks + to, 1, block), dtype=torch.int32, device="cuda")
    position[perm[:blocks].long(), 0] = torch.arange(blocks * block, device="cuda").view(blocks, block).to(torch.int32)
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")  # noqa: E731
    lens, out = i32(n), i32(0)
    ws = torch.empty(spf.spf_kv_evict_workspace_bytes(cache, to_table), dtype=torch.uint8, device="cuda")
    spf.spf_kv_evict(cache, spf.KvLedger(weight, position), lens, table, i32(keep), to_table, out, ws, n_first=5, n_recent=100)
    assert int(out) == keep
    flat = weight[table[0, :blocks].long(), 0].flatten()[:n].clone()
    flat[:5], flat[n - 100:] = float("inf"), float("inf")
    kept = flat.sort(descending=True, stable=True).indices[:keep].sort().values
    got = position[to_table[0].long(), 0].flatten()[:keep].long()
    assert torch.equal(got, kept)
    rows = pool[table[0, :blocks].long(), 0].flatten(0, 1)[kept]
    assert torch.equal(pool[to_table[0].long(), 0].flatten(0, 1)[:keep], rows)


def test_scales_of_an_8_bit_cache_far_apart():
    import paper_2603_02631_b200 as spf
    s = any_step(8, 2, 2, 64, 128, [640], [0], 5)
    gen = torch.Generator().manual_seed(6)
    for x in ("k_scale", "v_scale"):
        getattr(s, x).copy_(2.0 ** torch.randint(-20, 20, s.k_scale.shape, generator=gen).float())
    s.k_scale.mul_(1.3)                                    # not powers of two
    check(spf, s, 8, [200], 2, *ledger_of(s, 1))


def test_bad_places_are_reported():
    import paper_2603_02631_b200 as spf
    for what in ("length", "negative length", "source", "target"):
        s = any_step(4, 1, 1, 64, 128, [300, 300], [0, 0], 7)
        to = more_blocks(s, 4).view(2, 2).contiguous().cuda()
        weight, position = (torch.zeros((s.k_pool.shape[0], 1, 128), dtype=t, device="cuda") for t in (torch.float32, torch.int32))
        weight.copy_(torch.rand(weight.shape, generator=torch.Generator().manual_seed(1)))
        if what == "length":
            s.seq_lens[1] = 128 * s.table.shape[1] + 1
        elif what == "negative length":
            s.seq_lens[1] = -1
        elif what == "source":
            s.table[1, 1] = s.k_pool.shape[0]
        else:
            to[1, 1] = -1
        before = s.k_pool.clone()
        lens = cut(spf, s, weight, position, [200, 200], to, status=-7)
        assert lens.tolist() == [200, 0 if "length" in what else 200]
        assert not torch.equal(s.k_pool[to[0].long()], before[to[0].long()])
        others = [b for b in range(s.k_pool.shape[0]) if b not in to.flatten().tolist()]
        assert torch.equal(s.k_pool[others], before[others])


def test_random_cuts():
    import paper_2603_02631_b200 as spf
    rng = random.Random(8)
    for i in range(30):
        bits, d, Hkv, seqs = rng.choice([16, 8, 4]), rng.choice([64, 128]), rng.choice([1, 2, 5]), rng.randint(1, 4)
        lens = [rng.choice([0, 1, 63, 64, 100, 256, 391]) for _ in range(seqs)]
        keep = [rng.choice([0, 1, 64, 65, 200, 400]) for _ in range(seqs)]
        s = any_step(bits, Hkv, Hkv, d, 128, lens, [0] * seqs, i)
        weight, position = ledger_of(s, i)
        if rng.random() < 0.3:
            weight = weight.round()
        check(spf, s, bits, keep, rng.randint(1, 4), weight, position if rng.random() < 0.5 else None, rng.choice([0, 4]), rng.choice([0, 30, 300]))


def test_values_survive():
    """What attention reads of a kept token is what it read before (8 bits: rounded to the group's scale)."""
    import paper_2603_02631_b200 as spf
    for bits in (16, 8, 4):
        s = any_step(bits, 1, 1, 64, 128, [256], [0], 9)
        full = values_of(bits, s.v_pool, s.v_scale)[s.table[0].long().cpu(), 0].flatten(0, 1)[:256]
        weight, _ = ledger_of(s, 1)
        to = more_blocks(s, 2).view(1, 2).contiguous().cuda()
        weight = torch.cat([weight, torch.zeros((2, 1, 128), device="cuda")])
        position = torch.zeros(weight.shape, dtype=torch.int32, device="cuda")
        position[s.table[0].long(), 0] = torch.arange(256, dtype=torch.int32, device="cuda").view(2, 128)
        cut(spf, s, weight, position, [150], to)
        got = values_of(bits, s.v_pool, s.v_scale)[to[0].long().cpu(), 0].flatten(0, 1)[:150]
        want = full[position[to[0].long(), 0].flatten()[:150].long().cpu()]
        slack = torch.zeros_like(want) if bits != 8 else 2.0 ** -10 * s.v_scale.max().double().cpu() + want.abs() * 2.0 ** -4
        assert ((got - want).abs() <= slack).all()
