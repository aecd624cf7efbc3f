"""The 64-bit reference of the cache's attention for long sequences and many rows: whole heads at a time, on the GPU.  The formulas and
the bounds are those of kv_reference.attention and of test_gpu_attend.compare."""
import math

import torch

from kv_reference import SCALE_TOKENS, Step


def gpu_step(Hq, Hkv, d, block, old, new, bits, seed=0, rows=None, q_scale=1.0):
    """kv_reference.make_step for long sequences: the pools are made on the GPU, block by block in random order.  Groups of 64 tokens
    differ in magnitude by powers of two."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = [a + b for a, b in zip(old, new)]
    need = [-(-n // block) for n in lens]
    blocks = sum(need) + 2
    perm = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(old), max(need)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b]) + n]
    pools, scales = [], []
    for _ in range(2):
        x = torch.randn((blocks, Hkv, block // SCALE_TOKENS, SCALE_TOKENS, d), generator=gen, device="cuda")
        x *= 2.0 ** torch.randint(-2, 3, (blocks, Hkv, block // SCALE_TOKENS, 1, 1), generator=gen, device="cuda").float()
        if bits == 16:
            pools.append(x.view(blocks, Hkv, block, d).to(torch.bfloat16))
            scales.append(None)
            continue
        scale = 2.0 ** torch.ceil(torch.log2(x.abs().amax((-1, -2)) / 448.0))
        pools.append((x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(blocks, Hkv, block, d))
        scales.append(scale)
    n_rows = sum(new) if rows is None else rows
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    q = (torch.randn((n_rows, Hq, d), generator=gen, device="cuda") * q_scale).to(torch.bfloat16)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return Step(Hq, Hkv, d, block, list(old), list(new), n_rows, pools[0], pools[1], scales[0], scales[1], table, i32(starts), i32(lens), q, None, None)


def decoded(pool, scale, table_row, head, n):
    """float64 [n, d]: one head's keys or values of a sequence in order."""
    ids = table_row[:-(-n // pool.shape[2])].long()
    x = pool[ids, head]
    if scale is None:
        return x.double().flatten(0, 1)[:n]
    s = scale[ids, head].double().repeat_interleave(SCALE_TOKENS, -1)[..., None]
    return (x.view(torch.float8_e4m3fn).float().double() * s).flatten(0, 1)[:n]


def reference(s, b, head, first=0, causal=True, scale=None, tokens=None):
    """(out, lse, weight, terms) of some of a sequence's new tokens (all: None) and the query heads of a key head: float64
    [tokens, heads, d], [tokens, heads], sum p |v|, and the largest sum |scale q k| of a row's logits."""
    group, n, new = s.Hq // s.Hkv, s.old[b] + s.new[b], s.new[b]
    tokens = torch.arange(new, device="cuda") if tokens is None else tokens
    k, v = decoded(s.k_pool, s.k_scale, s.table[b], head, n), decoded(s.v_pool, s.v_scale, s.table[b], head, n)
    q = s.q[int(s.row_start[b]) + tokens][:, head * group:(head + 1) * group].double()
    scale = 1.0 / math.sqrt(s.d) if scale is None else scale
    key = torch.arange(n, device="cuda")
    hidden = (key < first)[None, :].expand(len(tokens), -1)
    if causal:
        hidden = hidden | (key[None, :] > (n - new + tokens)[:, None])
    z = torch.einsum("tgd,nd->tgn", q, k) * scale
    z.masked_fill_(hidden[:, None], -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total))[..., 0]
    p /= torch.where(total > 0, total, torch.ones_like(total))
    terms = torch.einsum("tgd,nd->tgn", q.abs(), k.abs()).mul_(scale).masked_fill_(hidden[:, None], 0.0).amax(-1)
    return torch.einsum("tgn,nd->tgd", p, v), lse, torch.einsum("tgn,nd->tgd", p, v.abs()), terms


def check(s, out, lse, causal=True, first=None, scale=None, heads=None, tokens=None, operand=None):
    """Compares rows of every sequence with the reference.  Tolerances as derived in test_gpu_attend.compare: a logit is an fp32 sum
    of exact products, off by less than 2^-16 sum |scale q k|; weights by that twice (the sum of them has it too), by ex2's 2^-21 and by
    half a step of the second product's operands (bf16 2^-8, fp16 2^-11); the output by half a step of bf16."""
    if operand is None:
        operand = 2.0 ** -8 if s.k_scale is None else 2.0 ** -11
    group = s.Hq // s.Hkv
    for b, new in enumerate(s.new):
        if new == 0:
            continue
        at = torch.arange(new, device="cuda") if tokens is None else tokens[tokens < new]
        row = int(s.row_start[b]) + at
        for h in range(s.Hkv) if heads is None else heads:
            part = slice(h * group, (h + 1) * group)
            want, want_lse, weight, terms = reference(s, b, h, 0 if first is None else first[b], causal, scale, at)
            off = terms * 2.0 ** -16 + 2.0 ** -20
            got, got_lse = out[row][:, part].double(), lse[row][:, part].double()
            empty = want_lse == -math.inf
            assert torch.equal(got_lse == -math.inf, empty), (b, h)
            assert (got[empty] == 0).all(), (b, h)
            d_lse = ((got_lse - want_lse).abs() - off - 2.0 ** -22 * want_lse.abs())[~empty]
            assert (d_lse <= 0).all(), (b, h, float(d_lse.max()))
            bound = 2.0 ** -8 * want.abs() + (operand + 2 * off[..., None]) * weight * (1 + 2.0 ** -8)
            d_out = (got - want).abs() - bound
            assert (d_out <= 0).all(), (b, h, float(d_out.max()))
