"""Outputs that overlap a call's inputs are refused, slices of one buffer that lie between one another are not (no GPU: a call that
gets past the checks ends with SPF_ERR_CUDA)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CALLS = """
import ctypes, random
import paper_2603_02631_b200 as spf
from paper_2603_02631_b200 import binding as b

P, D = 1 << 20, 64
ref = lambda x: None if x is None else ctypes.byref(x)
cache = b._KvCache(P << 8, P << 8, None, None, 10, 256, 2, D)


def attend(rows, q, out, heads=4):
    step = b._KvStep(1, rows, 1, 3, P, P, P)
    return spf.lib.spf_attend(ref(cache), ref(step), ref(q), ref(out), heads, 0.0, None, 256, 1 << 40, None, None)


def append(rows, q, q_out, k, v, heads=4):
    step = b._KvStep(1, rows, 1, 3, P, P, P)
    return spf.lib.spf_kv_append(ref(cache), ref(step), None, ref(k), ref(v), ref(q), ref(q_out), heads, None, None)


def at(element, row, head):
    return b._Rows(P + 2 * element, row, head)


def elements(r, rows, heads):
    start = (r.data - P) // 2
    return {start + i * r.stride_row + h * r.stride_head + j for i in range(rows) for h in range(heads) for j in range(0, D, 8)}


# slices of a fused buffer of 12 heads: queries, outputs, keys, values
fused = lambda head: at(head * D, 12 * D, D)
far = at(1 << 22, 4 * D, D)
assert attend(50, fused(0), fused(4)) == -4 and attend(50, fused(4), fused(0)) == -4, spf.spf_last_error()
assert attend(50, fused(0), fused(0)) == -1 and attend(50, fused(0), fused(3)) == -1 and attend(50, fused(3), fused(0)) == -1
assert attend(50, fused(9), fused(0)) == -1 and "overlaps" in spf.spf_last_error()      # its last head is the next row's first
assert attend(1, fused(9), fused(0)) == -4                                              # there is no next row
assert append(50, fused(0), fused(0), fused(4), fused(6)) == -4                         # in place
assert append(50, fused(0), fused(8), fused(4), fused(6)) == -4
assert append(50, fused(0), fused(1), fused(6), fused(8)) == -1 and "q" in spf.spf_last_error()
assert append(50, fused(0), fused(5), fused(4), fused(9)) == -1 and "k or v" in spf.spf_last_error()
assert append(50, fused(0), fused(5), fused(9), fused(4)) == -1
assert append(50, fused(0), at(0, 24 * D, D), far, far) == -1                           # in place with other strides
# heads outside: [heads][rows][d], and one lookahead token of [heads][m][d]
assert attend(50, at(0, D, 50 * D), at(4 * 50 * D, D, 50 * D)) == -4
assert attend(50, at(0, D, 50 * D), at(3 * 50 * D, D, 50 * D)) == -1
assert attend(3, at(0, 4 * 8 * D, 8 * D), at(5 * D, 4 * 8 * D, 8 * D)) == -4
assert attend(3, at(0, 4 * 8 * D, 8 * D), at(0, 4 * 8 * D, 8 * D)) == -1
# queries that are one row for all
assert attend(50, at(0, 0, D), at(4 * D, 4 * D, D)) == -4 and attend(50, at(60 * D, 0, D), at(0, 4 * D, D)) == -1

# against a look at every element
rng = random.Random(1)
seen = set()
for _ in range(4000):
    rows, heads = rng.randint(1, 6), rng.choice([2, 4])
    def layout():
        if rng.random() < 0.5:
            return rng.choice([heads, heads + 1, 2 * heads, 12]) * D + rng.choice([0, 8]), D + rng.choice([0, 0, 0, 8, 64])
        return D + rng.choice([0, 8]), (rows + rng.randint(0, 3)) * (D + 8)
    a, o = layout(), layout()
    if rng.random() < 0.5:
        o = a
    q, out = at(rng.randrange(0, 4000, 8), *a), at(rng.randrange(0, 4000, 8), *o)
    meet = bool(elements(q, rows, heads) & elements(out, rows, heads))
    got = attend(rows, q, out, heads)
    assert got == (-1 if meet else -4), (rows, heads, q.data, a, out.data, o, got, spf.spf_last_error())
    if not (q.data == out.data and a == o):
        assert append(rows, q, out, far, far, heads) == got, (rows, heads, q.data, a, out.data, o)
    seen.add((meet, a == o))
assert len(seen) == 4
"""


def test_overlaps():
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")       # the pointers are made up: no device may be reached
    proc = subprocess.run([sys.executable, "-c", CALLS], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, proc.stderr[-2000:]
