"""spf_attend where a CTA works through many key tiles and several (sequence, row tile, key head) triples: the ring's rounds, references
that move between tiles, queries reloaded, parts that begin and end inside a triple, triples of several tiles written whole."""
import pytest
import torch

from attend_reference import check, gpu_step
from test_gpu_attend import run

pytestmark = pytest.mark.gpu

CTAS, DEEPEST = 444, 8      # the most CTAs of a launch (three on each of 148 SMs), the most stages of a ring


def rising(s, steep):
    """Adds a channel to keys and queries that makes logits rise along the keys of even sequences and fall along those of odd ones, by
    `steep` in all (natural), so that rows' references move again and again."""
    for b, (old, new) in enumerate(zip(s.old, s.new)):
        n = old + new
        pos = torch.arange(n, device="cuda")
        ramp = pos.float() / n if b % 2 == 0 else 1 - pos.float() / n
        blocks, place = s.table[b].long()[pos // s.block], pos % s.block
        if s.k_scale is None:
            s.k_pool[blocks, :, place, 3] = (2 * ramp)[:, None].to(torch.bfloat16)
        else:
            scale = s.k_scale[blocks, :, place // 64]
            s.k_pool[blocks, :, place, 3] = (2 * ramp[:, None] / scale).clamp(max=448).to(torch.float8_e4m3fn).view(torch.uint8)
    s.q[..., 3] = steep * s.d ** 0.5 / 2


# rows of a key head up to 8, 16 and 32 (one token, two, four; eight heads a group of which there are 8), both dimensions
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,new", [(8, 8, 64, 1), (16, 8, 128, 1), (64, 8, 64, 1), (32, 8, 128, 3), (32, 8, 64, 8), (32, 8, 128, 8)])
@pytest.mark.parametrize("steep", [0, 40])
def test_few_rows_over_many_tiles(Hq, Hkv, d, new, steep, bits):
    import paper_2603_02631_b200 as spf
    old = [16001, 14000, 15203, 16383, 14464, 15999, 14333, 16000]
    assert sum(Hkv * (n // 128) for n in old) > 2 * DEEPEST * CTAS
    s = gpu_step(Hq, Hkv, d, 256, old, [new] * 8, bits, seed=Hq + d + new)
    if steep:
        rising(s, steep)
    check(s, *run(spf, s), heads=[0, 3, 7])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (4, 2, 128), (24, 8, 128), (16, 16, 64)])
def test_few_rows_over_many_short_sequences(Hq, Hkv, d, bits):
    """Triples of one to five tiles, many to a CTA."""
    import paper_2603_02631_b200 as spf
    old = [(149 * b) % 600 for b in range(900)]
    new = [1 + (b % 7 == 0) - (b % 11 == 3) for b in range(900)]
    s = gpu_step(Hq, Hkv, d, 128, old, new, bits, seed=Hq)
    out, lse = run(spf, s)
    s.new = [n if b % 9 == 0 or b > 890 else 0 for b, n in enumerate(new)]       # those that are compared
    s.old = [a + n - m for a, n, m in zip(old, new, s.new)]
    check(s, out, lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,old,new", [
    (16, 8, 64, [9000, 100], [1001, 1500]),                  # a CTA has some 60 tiles
    (16, 8, 128, [9000, 100], [1001, 1500]),
    (16, 4, 128, [0, 0], [4100, 2049]),                      # whole prompts from their first token
    (8, 1, 64, [0], [9000]),
    (6, 2, 128, [3000, 0, 500, 7, 6000], [300, 1, 700, 0, 90]),
])
@pytest.mark.parametrize("steep", [0, 40])
def test_many_rows_over_many_tiles(Hq, Hkv, d, old, new, steep, bits):
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 256, old, new, bits, seed=sum(new))
    if steep:
        rising(s, steep)
    out, lse = run(spf, s)
    tokens = torch.unique(torch.cat([torch.arange(0, max(new), 37), torch.arange(max(new) - 3, max(new)), torch.arange(3),
                                     torch.tensor([127, 128, 129, 255, 256, 257, 299, 699, 1000, 1499, 2048])])).cuda()
    check(s, out, lse, heads=sorted({0, Hkv // 2, Hkv - 1}), tokens=tokens)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_of_many_sequences(d, bits):
    """More sequences than the kernel for many rows has threads, most of them short, some without tokens."""
    import paper_2603_02631_b200 as spf
    old = [(97 * b) % 300 for b in range(1100)]
    new = [0 if b % 13 == 5 else 1 + (b * 31) % 60 for b in range(1100)]
    s = gpu_step(4, 2, d, 128, old, new, bits, seed=3)
    out, lse = run(spf, s, max_new=60)
    s.new = [n if b % 17 == 0 or b > 1095 else 0 for b, n in enumerate(new)]
    s.old = [a + n - m for a, n, m in zip(old, new, s.new)]
    check(s, out, lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,old,new", [(32, 8, 64, [14000] * 6, [8] * 6), (16, 8, 128, [14000] * 6, [2] * 6), (16, 8, 64, [6000, 0], [700, 2000]), (16, 8, 128, [6000, 0], [700, 2000])])
def test_values_that_are_not_finite_in_long_sequences(Hq, Hkv, d, old, new, bits):
    """NaN in the value of a new token: the rows from it on have NaN in that dimension and nothing else changes."""
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 128, old, new, bits, seed=9)
    clean, clean_lse = run(spf, s)
    b, head, dim, at = len(old) - 1, 5, d - 7, new[-1] // 2
    pos = old[b] + at
    s.v_pool[int(s.table[b, pos // 128]), head, pos % 128, dim] = float("nan") if bits == 16 else 0x7F
    out, lse = run(spf, s)
    group, first = Hq // Hkv, int(s.row_start[b])
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[first + at:first + new[b], head * group:(head + 1) * group, dim] = True
    assert out[hit].isnan().all()
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,old,new", [(16, 8, 128, [14000] * 6, [1] * 6), (32, 8, 64, [14000] * 6, [8] * 6), (16, 8, 128, [6000, 0], [700, 2000]), (16, 8, 64, [6000, 0], [700, 2000])])
def test_first_keys_and_all_keys_over_many_tiles(Hq, Hkv, d, old, new, bits):
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 128, old, new, bits, seed=10)
    first = [(old[b] + new[b]) * (b + 1) // (len(old) + 1) + b for b in range(len(old))]
    tokens = torch.unique(torch.cat([torch.arange(0, max(new), 61), torch.tensor([first[-1] - old[-1] - 1, first[-1] - old[-1], first[-1] - old[-1] + 1])
                                     .clamp(0, max(new) - 1)])).cuda()
    for causal in (True, False):
        out, lse = run(spf, s, causal=causal, first=first)
        check(s, out, lse, causal=causal, first=first, heads=[1, 6], tokens=tokens)


@pytest.mark.parametrize("bits", [16, 8])
def test_repeated_calls_give_the_same_bits(bits):
    import paper_2603_02631_b200 as spf
    for s in (gpu_step(16, 8, 128, 256, [14000] * 4, [1] * 4, bits, seed=11), gpu_step(32, 8, 64, 256, [30000], [8], bits, seed=12),
              gpu_step(16, 8, 64, 256, [5000, 10], [600, 900], bits, seed=13)):
        clean = run(spf, s)
        for _ in range(5):
            again = run(spf, s)
            assert torch.equal(clean[0], again[0]) and torch.equal(clean[1], again[1])
