"""Plain 64-bit reference of caches in 4 bits (codes 0 ... 15, two to a byte, a bf16 scale for 32 dimensions of a token), and steps to try
them on.  Everything on the CPU."""
import math

import torch

from kv_reference import Step, make_step

SCALE_DIMS = 32


def values(pool, scale):
    """float64 [..., d] of codes and scales."""
    pool, scale = pool.cpu(), scale.cpu().double()
    x = torch.stack([pool & 15, pool >> 4], -1).flatten(-2).double() - 8
    return x * scale.repeat_interleave(SCALE_DIMS, -1)


def sizes(scale):
    """float64 [..., d]: 23 scales, which bounds what a code and the 8 subtracted from it are worth, one by one."""
    return 23 * scale.cpu().double().repeat_interleave(SCALE_DIMS, -1)


def short_scale(amax: float) -> float:
    """The smallest number of five significant bits s >= 2^-100 with 7 s >= amax."""
    if amax <= 7 * 2.0 ** -100:
        return 2.0 ** -100
    e = math.floor(math.log2(amax / 7)) - 4
    m = math.floor(amax / 7 / 2.0 ** e) - 1
    while 7 * m * 2.0 ** e < amax:
        m += 1
    while m > 32 and 7 * (m // 2) * 2.0 ** (e + 1) >= amax:
        m, e = m // 2, e + 1
    return m * 2.0 ** e if m <= 32 else math.ceil(m / 2) * 2.0 ** (e + 1)


def random_pool4(gen, n_blocks, Hkv, block, d, spread=2):
    """Codes of every value, and scales that differ by powers of two and have up to five significant bits."""
    pool = torch.randint(0, 256, (n_blocks, Hkv, block, d // 2), generator=gen).to(torch.uint8)
    shape = (n_blocks, Hkv, block, d // SCALE_DIMS)
    scale = torch.randint(16, 32, shape, generator=gen) * 2.0 ** torch.randint(-spread - 6, spread - 5, shape, generator=gen).float()
    return pool, scale.to(torch.bfloat16)


def make_step4(Hq, Hkv, d, block, old, new, seed=0, behind=0, device="cuda", fused=True):
    """kv_reference.make_step with pools of 4 bits."""
    s = make_step(Hq, Hkv, d, block, old, new, 16, seed, behind, device, fused)
    gen = torch.Generator().manual_seed(seed + 1)
    n_blocks = s.k_pool.shape[0]
    for x in "kv":
        pool, scale = random_pool4(gen, n_blocks, Hkv, block, d)
        setattr(s, x + "_pool", pool.to(device))
        setattr(s, x + "_scale", scale.to(device))
    return s


def logical4(pool, scale, table_row, n):
    """float64 [heads, n, d] twice: a sequence's keys or values in order, and the sizes of what they are made of."""
    ids = table_row[:-(-n // pool.shape[2])].long().cpu() if n else torch.zeros(0, dtype=torch.long)
    flat = lambda x: x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n]  # noqa: E731
    return flat(values(pool.cpu()[ids], scale.cpu()[ids])), flat(sizes(scale.cpu()[ids]))


def attention4(s: Step, b, first=0, causal=True, scale=None):
    """(out, lse, weight, wide, terms) of the new tokens of sequence b: float64 [tokens, heads, d] and [tokens, heads]; weight: sum p |v|,
    wide: sum p times the sizes of the values' parts, terms: the largest sum |scale q| times those of the keys'."""
    n, new, row, group = s.old[b] + s.new[b], s.new[b], int(s.row_start[b]), s.Hq // s.Hkv
    scale = 1.0 / math.sqrt(s.d) if scale is None else scale
    (k, k_size), (v, v_size) = logical4(s.k_pool, s.k_scale, s.table[b], n), logical4(s.v_pool, s.v_scale, s.table[b], n)
    q = s.q[row:row + new].double().cpu()
    shape = (new, s.Hq, s.d)
    out, weight, wide = (torch.zeros(shape, dtype=torch.float64) for _ in range(3))
    lse, terms = torch.full((new, s.Hq), -math.inf, dtype=torch.float64), torch.zeros((new, s.Hq), dtype=torch.float64)
    key = torch.arange(n)
    pos = s.old[b] + torch.arange(new)
    hidden = (key < first)[None, :].expand(new, -1)
    if causal:
        hidden = hidden | (key[None, :] > pos[:, None])
    for h in range(s.Hq):
        g = h // group
        z = (q[:, h] @ k[g].T * scale).masked_fill(hidden, -math.inf)
        lse[:, h] = torch.logsumexp(z, -1)
        p = torch.exp(z - lse[:, h, None]).masked_fill(hidden, 0.0)
        out[:, h] = torch.where(p[..., None] > 0, p[..., None] * v[g][None], torch.zeros(1, dtype=torch.float64)).sum(1)
        weight[:, h], wide[:, h] = p @ v[g].abs(), p @ v_size[g]
        if n:
            terms[:, h] = (q[:, h].abs() @ k_size[g].T * scale).masked_fill(hidden, 0.0).amax(-1)
    return out, lse, weight, wide, terms


def compare4(s, out, lse, causal=True, first=None, scale=None, seqs=None, fill=7.0):
    """Tolerances.  A logit is an fp32 sum of exact products and exact scales: at most 128 + 4 roundings of 2^-24 (2^-23 where the unit cuts off)
    of partial sums that `terms` bounds, below 2^-15 terms with the factor's; the weights are off by that twice (their sum has it too), by
    ex2's 2^-21, and by half a step of bf16 where scales go into them (few rows) or where they are rounded (many); sums of n values are fp32:
    n 2^-23 of `wide`, n below 2^10; the output is rounded to bf16."""
    for b, new in enumerate(s.new):
        if new == 0 or (seqs is not None and b not in seqs):
            continue
        rows = slice(int(s.row_start[b]), int(s.row_start[b]) + new)
        want, want_lse, weight, wide, terms = attention4(s, b, 0 if first is None else max(first[b], 0), causal, scale)
        off = terms * 2.0 ** -15 + 2.0 ** -20
        got, got_lse = out[rows].double().cpu(), lse[rows].double().cpu()
        empty = want_lse == -math.inf
        assert torch.equal(got_lse == -math.inf, empty), b
        assert (got[empty] == 0).all(), b
        d_lse = ((got_lse - want_lse).abs() - off - 2.0 ** -22 * want_lse.abs())[~empty]
        assert (d_lse <= 0).all(), (b, float(d_lse.max()))
        bound = 2.0 ** -8 * want.abs() + ((2.0 ** -8 + 2 * off[..., None]) * weight + 2.0 ** -13 * wide) * (1 + 2.0 ** -8)
        d_out = (got - want).abs() - bound
        assert (d_out <= 0).all(), (b, float(d_out.max()))
    rows = sum(s.new)
    assert (out[rows:] == fill).all() and (lse[rows:] == fill).all()
