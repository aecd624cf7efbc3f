"""spf_kv_weigh over bf16 keys with infinite elements: a key that every row gives a logit of -inf receives nothing, whatever fills a tile up beside
the rows."""
import math

import pytest
import torch

from ledger_reference import ledger_of
from kv_reference import make_step
from test_gpu_kv_weigh import check, weigh

pytestmark = pytest.mark.gpu


def infinite_step(Hq, Hkv, d, block, old, new, seed):
    """Some keys (of the first tile, at its end, of the step itself) have an infinite element in dimension 5, where every query is negative."""
    s = make_step(Hq, Hkv, d, block, old, new, 16, seed, behind=1)
    s.q[..., 5] = -s.q[..., 5].abs() - 0.5
    for b, (o, n) in enumerate(zip(old, new)):
        for key in {0, min(63, o + n - 1), o // 2, o + n - 1}:
            s.k_pool[int(s.table[b, key // block]), :, key % block, 5] = math.inf
    return s


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (2, 2), (6, 2), (5, 1), (12, 2), (12, 1)])
@pytest.mark.parametrize("new", [[1], [1, 1, 1], [7, 2]])
def test_few_rows(Hq, Hkv, new):
    import paper_2603_02631_b200 as spf
    for d in (64, 128):
        check(spf, infinite_step(Hq, Hkv, d, 128, [200, 63, 130][:len(new)], new, d), 16, decay=0.5)


@pytest.mark.parametrize("max_new", [1, 9, None])
def test_the_last_tile_of_more_rows(max_new):
    import paper_2603_02631_b200 as spf
    check(spf, infinite_step(4, 2, 64, 128, [300], [27], 3), 16, decay=0.5, max_new=max_new)


def attend_and_weigh(Hq, Hkv, new):
    import paper_2603_02631_b200 as spf
    s = infinite_step(Hq, Hkv, 64, 128, [200], [new], 6)
    out, lse = torch.zeros(s.q.shape, dtype=torch.bfloat16, device="cuda"), torch.zeros((s.rows, Hq), device="cuda")
    ws = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), s.step(spf), s.q), dtype=torch.uint8, device="cuda")
    spf.spf_attend(s.cache(spf), s.step(spf), s.q, out, ws, lse)
    weight, _ = ledger_of(s, 5)
    weigh(spf, s, lse, weight, None)
    return [bool(torch.isfinite(x).all()) for x in (out[:new], lse[:new], weight)]


@pytest.mark.parametrize("Hq,Hkv,new", [(1, 1, 1), (6, 2, 5)])
def test_attention_and_what_follows_it(Hq, Hkv, new):
    """The attention leaves these rows finite, and so are the weights that are made with its log-sum-exps."""
    assert attend_and_weigh(Hq, Hkv, new) == [True] * 3


def test_a_row_that_saw_no_key_adds_nothing_to_keys_that_are_not_numbers():
    """Its log-sum-exp is -inf, which decides, whatever its products are."""
    import paper_2603_02631_b200 as spf
    for new in (1, 3):
        s = make_step(4, 2, 64, 128, [100], [new], 16, 7)
        s.k_pool[int(s.table[0, 0]), :, 40, 3], s.k_pool[int(s.table[0, 0]), :, 41, 3] = math.nan, math.inf
        lse = torch.full((s.rows, 4), -math.inf, device="cuda")
        weight, _ = ledger_of(s, 5)
        before = weight.clone()
        weigh(spf, s, lse, weight, None, decay=0.5)
        block = int(s.table[0, 0])
        assert torch.equal(weight[block, :, :100], before[block, :, :100] * 0.5) and (weight[block, :, 100:100 + new] == 0).all()


@pytest.mark.parametrize("Hq,Hkv", [(3, 1), (10, 2), (6, 1), (7, 1), (9, 1), (70, 1)])
@pytest.mark.parametrize("last", [0, 50])
def test_many_rows_of_heads_that_do_not_fill_a_tile(Hq, Hkv, last):
    """128 rows of a tile are as many tokens as fit whole: 3, 5, 6 ... heads leave columns without a row in each."""
    import paper_2603_02631_b200 as spf
    for d in (64, 128):
        check(spf, infinite_step(Hq, Hkv, d, 128, [200, 5], [170, 65], d), 16, decay=0.5, last=last)


def test_many_rows_of_which_some_saw_no_key():
    """As test_a_row_that_saw_no_key_adds_nothing_to_keys_that_are_not_numbers, in a chunk: keys 40 and 41 are seen by rows without keys only."""
    import paper_2603_02631_b200 as spf
    s = make_step(4, 2, 64, 128, [100], [130], 16, 7)
    s.k_pool[int(s.table[0, 0]), :, 40, 3], s.k_pool[int(s.table[0, 0]), :, 41, 3] = math.nan, math.inf
    lse = torch.full((s.rows, 4), -math.inf, device="cuda")
    weight, _ = ledger_of(s, 5)
    before = weight.clone()
    weigh(spf, s, lse, weight, None, decay=0.5)
    block, second = int(s.table[0, 0]), int(s.table[0, 1])
    assert torch.equal(weight[block, :, :100], before[block, :, :100] * 0.5) and (weight[block, :, 100:] == 0).all() and (weight[second, :, :102] == 0).all()


def test_attention_of_a_chunk_and_what_follows_it():
    assert attend_and_weigh(6, 2, 100) == [True] * 3
