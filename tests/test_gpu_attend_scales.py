"""spf_attend on 8-bit caches whose value scales span what the header allows, 2^-100 (the scale of values that are all zero) to 2^100:
the sum of the weights and the weighted values each need a reference of their own."""
import math

import pytest
import torch

from attend_reference import check, gpu_step
from test_gpu_attend import run

pytestmark = pytest.mark.gpu

ZERO = 2.0 ** -100                                          # what spf_kv_append gives to values that are all zero
LN2 = math.log(2.0)                                         # softmax_scale with which q . k are base-2 logits

# query heads, key heads, dimensions, new tokens: tiles of 8, 16 and 32 rows, and the kernel for many
FORMS = [(2, 1, 64, 1), (2, 1, 128, 1), (4, 1, 64, 4), (4, 1, 128, 4), (4, 1, 64, 8), (4, 1, 64, 40), (4, 1, 128, 40)]


def logical_tokens(s, b):
    """Pool block and place of every token of a sequence."""
    pos = torch.arange(s.old[b] + s.new[b], device="cuda")
    return s.table[b].long()[pos // s.block], pos % s.block


def set_logits(s, base2):
    """Every row's base-2 logits (with softmax_scale LN2) become `base2` [tokens], which has to consist of E4M3 numbers, plus one of
    -1, 0, 1 by token and row."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    s.q.zero_()
    s.q[..., 0] = 1.0
    s.q[..., 5] = torch.randint(-1, 2, s.q.shape[:2], generator=gen, device="cuda").to(torch.bfloat16)
    k = torch.zeros((len(base2), s.d), device="cuda")
    k[:, 0] = base2
    k[:, 5] = torch.randint(-1, 2, (len(base2),), generator=gen, device="cuda").float()
    raw = k.to(torch.float8_e4m3fn)
    assert torch.equal(raw.float(), k)
    blocks, place = logical_tokens(s, 0)
    s.k_pool[blocks, :, place] = raw.view(torch.uint8)[:, None]
    s.k_scale.fill_(1.0)


def set_value_scales(s, exponents):
    """The groups of 64 tokens of sequence 0 get value scales 2^exponents[group]."""
    blocks, place = logical_tokens(s, 0)
    s.v_scale[blocks[::64], :, place[::64] // 64] = (2.0 ** exponents.double()).float()[:, None]


def zero_values(s, n):
    """The first n tokens' values become zeros, with their scale."""
    blocks, place = logical_tokens(s, 0)
    s.v_pool[blocks[:n], :, place[:n]] = 0
    s.v_scale[blocks[:n:64], :, place[:n:64] // 64] = ZERO


@pytest.mark.parametrize("Hq,Hkv,d,new", FORMS)
def test_values_that_are_all_zero(Hq, Hkv, d, new):
    """A cache that was warmed up with zeros: equal logits, log-sum-exps of ln n."""
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 128, [20000], [new], 8, seed=1)
    s.k_pool.zero_()
    zero_values(s, 20000 + new)
    out, lse = run(spf, s)
    assert (out == 0).all()
    want = torch.log(20001.0 + torch.arange(new, device="cuda", dtype=torch.float64))[:, None]
    assert ((lse.double() - want).abs() <= 2.0 ** -20 + 2.0 ** -22 * want).all()


@pytest.mark.parametrize("Hq,Hkv,d,new", FORMS)
def test_zero_values_under_rising_logits(Hq, Hkv, d, new):
    """Logits that rise again and again by nearly the 8 by which they may exceed the reference, and in the end far beyond it; heads
    enough for a CTA to see several tiles of each."""
    import paper_2603_02631_b200 as spf
    s = gpu_step(24 * Hq, 24 * Hkv, d, 128, [12000], [new], 8, seed=2)
    base2 = torch.arange(12000 + new, device="cuda") // 128 % 4 * 2.0
    base2[11000:] = 80.0
    set_logits(s, base2)
    zero_values(s, 12000 + new)
    out, lse = run(spf, s, scale=LN2)
    assert (out == 0).all()
    check(s, out, lse, scale=LN2, heads=range(0, 24 * Hkv, 5))


@pytest.mark.parametrize("Hq,Hkv,d,new", FORMS)
@pytest.mark.parametrize("zeros", [64, 5120, 11008])
def test_a_prefix_of_zero_values_before_ordinary_ones(Hq, Hkv, d, new, zeros):
    import paper_2603_02631_b200 as spf
    s = gpu_step(24 * Hq, 24 * Hkv, d, 128, [12000], [new], 8, seed=3)
    zero_values(s, zeros)
    check(s, *run(spf, s), heads=range(0, 24 * Hkv, 5))
    set_logits(s, torch.arange(12000 + new, device="cuda") // 128 % 4 * 2.0)
    check(s, *run(spf, s, scale=LN2), scale=LN2, heads=range(0, 24 * Hkv, 5))


@pytest.mark.parametrize("Hq,Hkv,d,new", FORMS)
def test_value_scales_over_the_whole_range(Hq, Hkv, d, new):
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 128, [9000], [new], 8, seed=4)
    gen = torch.Generator(device="cuda").manual_seed(5)
    groups = -(-(9000 + new) // 64)
    set_value_scales(s, torch.randint(-100, 101, (groups,), generator=gen, device="cuda"))
    check(s, *run(spf, s))
    set_value_scales(s, torch.randint(0, 2, (groups,), generator=gen, device="cuda") * 200 - 100)
    check(s, *run(spf, s))


@pytest.mark.parametrize("Hq,Hkv,d,new", FORMS)
@pytest.mark.parametrize("above", [0.0, 60.0, 144.0, 208.0, 320.0])
@pytest.mark.parametrize("order", ["small first", "large first", "in turns", "within a tile"])
def test_small_values_with_the_larger_logits(Hq, Hkv, d, new, above, order):
    """Groups of scale 2^-100 whose logits are `above` higher than those of scale 2^100: which of them the output and which the
    log-sum-exp consists of differs."""
    import paper_2603_02631_b200 as spf
    n = 6000 + new
    s = gpu_step(Hq, Hkv, d, 128, [6000], [new], 8, seed=6)
    group = torch.arange(-(-n // 64), device="cuda")
    small = {"small first": group < 40, "large first": group >= 40, "in turns": group // 8 % 2 == 0, "within a tile": group % 2 == 0}[order]
    set_value_scales(s, torch.where(small, -100, 100))
    set_logits(s, torch.where(small.repeat_interleave(64)[:n], above, 0.0))
    out, lse = run(spf, s, scale=LN2)
    check(s, out, lse, scale=LN2)
