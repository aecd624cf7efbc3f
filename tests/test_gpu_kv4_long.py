"""Caches of 4 bits and the ledger where a CTA works through many key tiles and several sequences: against 64 bits, whole heads at a time on the GPU."""
import math

import pytest
import torch

from kv4_reference import SCALE_DIMS
from kv_reference import SCALE_TOKENS, Step

pytestmark = pytest.mark.gpu


def gpu_step4(Hq, Hkv, d, block, old, new, bits=4, seed=0, q_scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = [a + b for a, b in zip(old, new)]
    need = [-(-n // block) for n in lens]
    blocks = sum(need) + 1
    perm = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(old), max(need)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b]) + n]
    pools, scales = [], []
    for _ in range(2):
        if bits == 4:
            pools.append(torch.randint(0, 256, (blocks, Hkv, block, d // 2), generator=gen, device="cuda").to(torch.uint8))
            shape = (blocks, Hkv, block, d // SCALE_DIMS)
            scales.append((torch.randint(16, 32, shape, generator=gen, device="cuda") * 2.0 ** torch.randint(-9, -5, shape, generator=gen, device="cuda").float())
                          .to(torch.bfloat16))
        elif bits == 8:
            pools.append(torch.randn((blocks, Hkv, block, d), generator=gen, device="cuda").mul_(64).to(torch.float8_e4m3fn).view(torch.uint8))
            scales.append(2.0 ** torch.randint(-8, -4, (blocks, Hkv, block // SCALE_TOKENS), generator=gen, device="cuda").float())
        else:
            pools.append(torch.randn((blocks, Hkv, block, d), generator=gen, device="cuda").to(torch.bfloat16))
            scales.append(None)
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    q = (torch.randn((sum(new), Hq, d), generator=gen, device="cuda") * q_scale).to(torch.bfloat16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return Step(Hq, Hkv, d, block, list(old), list(new), sum(new), pools[0], pools[1], scales[0], scales[1], table, i32(starts), i32(lens), q, None, None)


def decoded(s, bits, x, b, head, n):
    """float64 [n, d]: one head's keys or values, and the sizes of the parts they are made of."""
    pool, scale = getattr(s, x + "_pool"), getattr(s, x + "_scale")
    ids = s.table[b][:-(-n // s.block)].long()
    p = pool[ids, head]
    if bits == 16:
        v = p.double().flatten(0, 1)[:n]
        return v, v.abs()
    if bits == 8:
        v = (p.view(torch.float8_e4m3fn).float().double() * scale[ids, head].double().repeat_interleave(SCALE_TOKENS, -1)[..., None]).flatten(0, 1)[:n]
        return v, v.abs()
    wide = scale[ids, head].double().repeat_interleave(SCALE_DIMS, -1)
    v = torch.stack([p & 15, p >> 4], -1).flatten(-2).double() - 8
    return (v * wide).flatten(0, 1)[:n], (23 * wide).flatten(0, 1)[:n]


CASES = [(16, 2, 128, 1024, [60000], [1]), (16, 8, 128, 4096, [9000] * 12, [1] * 12), (8, 1, 64, 256, [70001, 33], [4, 4]), (4, 1, 128, 128, [30000], [3]),
         (8, 2, 64, 4096, [3000, 0], [900, 700]), (3, 1, 128, 512, [9000], [513])]


@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", CASES)
def test_attention_and_received_weights(Hq, Hkv, d, block, old, new):
    """Tolerances as in kv4_reference.compare4 and ledger_reference.received; fp32 sums over n keys are off by 2^-24 sqrt(n) of their sizes, here taken as
    2^-13 as there (n below 2^17, over many warps and CTAs)."""
    import paper_2603_02631_b200 as spf
    s = gpu_step4(Hq, Hkv, d, block, old, new, seed=d + len(old))
    group, step = Hq // Hkv, s.step(spf)
    out, lse = torch.zeros_like(s.q), torch.zeros((s.rows, Hq), device="cuda")
    ws = torch.empty(spf.spf_attend_workspace_bytes(s.cache(spf), step, s.q), dtype=torch.uint8, device="cuda")
    spf.spf_attend(s.cache(spf), step, s.q, out, ws, lse)
    weight = torch.rand(s.k_pool.shape[:3], device="cuda")
    before = weight.clone()
    spf.spf_kv_weigh(s.cache(spf), step, s.q, lse, spf.KvLedger(weight), decay=0.5)
    for b, (o, n_new) in enumerate(zip(old, new)):
        n, row = o + n_new, int(s.row_start[b])
        key = torch.arange(n, device="cuda")
        hidden = key[None, :] > (o + torch.arange(n_new, device="cuda"))[:, None]
        at, place = s.table[b].long()[key // block], key % block
        for h in range(Hkv):
            (k, k_size), (v, v_size) = decoded(s, 4, "k", b, h, n), decoded(s, 4, "v", b, h, n)
            got, slack = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
            for g in range(h * group, (h + 1) * group):
                q = s.q[row:row + n_new, g].double()
                z = (q @ k.T / math.sqrt(d)).masked_fill_(hidden, -math.inf)
                want_lse = torch.logsumexp(z, -1)
                p = torch.exp(z - want_lse[:, None])
                terms = (q.abs() @ k_size.T / math.sqrt(d)).masked_fill_(hidden, 0.0)
                off = terms.amax(-1) * 2.0 ** -15 + 2.0 ** -20
                assert ((lse[row:row + n_new, g].double() - want_lse).abs() <= off + 2.0 ** -22 * want_lse.abs()).all()
                want = p @ v
                bound = 2.0 ** -8 * want.abs() + ((2.0 ** -8 + 2 * off[:, None]) * (p @ v.abs()) + 2.0 ** -13 * (p @ v_size)) * (1 + 2.0 ** -8)
                assert ((out[row:row + n_new, g].double() - want).abs() <= bound).all()
                own = torch.exp(z - lse[row:row + n_new, g].double()[:, None])
                got += own.sum(0)
                slack += (own * (terms * 2.0 ** -15 + want_lse.abs()[:, None] * 2.0 ** -22 + 2.0 ** -20)).sum(0)
            want = torch.where(key < o, before[at, h, place].double() * 0.5, 0.0) + got
            assert ((weight[at, h, place].double() - want).abs() <= slack + 2.0 ** -20 * got + 2.0 ** -22 * want).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("Hq,Hkv,d,block,old,new", [(16, 8, 128, 4096, [9000] * 6, [1] * 6), (8, 2, 64, 4096, [3000, 0, 5000], [900, 700, 2]), (32, 2, 64, 256, [20000], [8])])
def test_received_weights_of_the_other_formats(Hq, Hkv, d, block, old, new, bits):
    import paper_2603_02631_b200 as spf
    s = gpu_step4(Hq, Hkv, d, block, old, new, bits, seed=d)
    group, step = Hq // Hkv, s.step(spf)
    lse = torch.full((s.rows, Hq), 3.0, device="cuda")             # any number will do
    weight = torch.zeros(s.k_pool.shape[:3], device="cuda")
    spf.spf_kv_weigh(s.cache(spf), step, s.q, lse, spf.KvLedger(weight))
    for b, (o, n_new) in enumerate(zip(old, new)):
        n, row = o + n_new, int(s.row_start[b])
        key = torch.arange(n, device="cuda")
        hidden = key[None, :] > (o + torch.arange(n_new, device="cuda"))[:, None]
        at, place = s.table[b].long()[key // block], key % block
        for h in range(Hkv):
            k, k_size = decoded(s, bits, "k", b, h, n)
            got, slack = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
            for g in range(h * group, (h + 1) * group):
                q = s.q[row:row + n_new, g].double()
                own = torch.exp((q @ k.T / math.sqrt(d)).masked_fill_(hidden, -math.inf) - 3.0)
                got += own.sum(0)
                slack += (own * ((q.abs() @ k_size.T / math.sqrt(d)) * 2.0 ** -15 + 2.0 ** -19)).sum(0)
            assert ((weight[at, h, place].double() - got).abs() <= slack + 2.0 ** -20 * got).all()


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_queries_with_rows_or_heads_for_all(bits):
    """Strides of zero (one row for every token, one head for every head; with many rows these are not what a copy of a box can read), rows that
    overlap, and heads outside."""
    import paper_2603_02631_b200 as spf
    s = gpu_step4(8, 2, 64, 256, [500], [90], bits, seed=1)
    lse = torch.full((s.rows, 8), 2.0, device="cuda")
    flat = s.q.contiguous().flatten()
    for q in (s.q[:1].expand(90, 8, 64), s.q[:, :1].expand(90, 8, 64), flat.as_strided((90, 8, 64), (8, 64, 1)), flat.as_strided((90, 8, 64), (64, 16, 1)),
              s.q.transpose(0, 1).contiguous().transpose(0, 1)):
        got = []
        for x in (q, q.contiguous()):
            weight = torch.zeros(s.k_pool.shape[:3], device="cuda")
            spf.spf_kv_weigh(s.cache(spf), s.step(spf), x, lse, spf.KvLedger(weight))
            got.append(weight)
        torch.cuda.synchronize()
        assert ((got[0] - got[1]).abs() <= 2.0 ** -16 * got[1]).all()


def test_more_heads_to_a_key_head_than_a_tile_has_rows():
    import paper_2603_02631_b200 as spf
    s = gpu_step4(130, 1, 64, 128, [200], [2], seed=2)
    lse = torch.full((2, 130), 1.0, device="cuda")
    weight = torch.zeros(s.k_pool.shape[:3], device="cuda")
    spf.spf_kv_weigh(s.cache(spf), s.step(spf), s.q, lse, spf.KvLedger(weight))
    k, k_size = decoded(s, 4, "k", 0, 0, 202)
    want, slack = torch.zeros(202, dtype=torch.float64, device="cuda"), torch.zeros(202, dtype=torch.float64, device="cuda")
    for t in range(2):
        own = torch.exp(s.q[t].double() @ k[:201 + t].T / 8 - 1.0)
        want[:201 + t] += own.sum(0)
        slack[:201 + t] += (own * (s.q[t].double().abs() @ k_size[:201 + t].T / 8 * 2.0 ** -15 + 2.0 ** -19)).sum(0)
    key = torch.arange(202, device="cuda")
    got = weight[s.table[0].long()[key // 128], 0, key % 128].double()
    assert ((got - want).abs() <= slack + 2.0 ** -20 * want).all()
