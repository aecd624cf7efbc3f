"""Up to 8 rows of a key head over a bf16 cache: weights keep 16 bits, so that next to the output's own rounding the fp32 logits alone
matter."""
import pytest

from attend_reference import check, gpu_step
from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,old,new", [(4, 2, 64, [20, 63, 300], [1, 1, 1]), (16, 2, 128, [20, 63, 300], [1, 1, 1]), (8, 8, 128, [9000], [8]), (8, 4, 64, [3, 40], [4, 2]),
                                              (32, 8, 128, [16000] * 4, [2] * 4)])
def test_weights_of_two_terms(Hq, Hkv, d, old, new):
    """Half a step of bf16, 2^-8, twice over: a weight is off by 2^-16."""
    import paper_2603_02631_b200 as spf
    s = gpu_step(Hq, Hkv, d, 128, old, new, 16, seed=d)
    check(s, *run(spf, s), operand=2.0 ** -16)
    if new[0] > 1:
        # the first token's row, where the value of the next one is infinite: products are then made row by row
        s.v_pool[int(s.table[0, (old[0] + 1) // 128]), 0, (old[0] + 1) % 128] = float("inf")
        out, lse = run(spf, s)
        s.new = [1] + [0] * (len(new) - 1)
        check(s, out, lse, operand=2.0 ** -16)
