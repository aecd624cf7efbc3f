"""Plain 64-bit reference of the ledger beside a cache (received attention weights) and of cuts to a budget.  Everything on the CPU."""
import math

import torch

from kv4_reference import logical4, make_step4, sizes, values
from kv_reference import SCALE_TOKENS, e4m3_values, logical, make_step


def any_step(bits, *args, **kwargs):
    return make_step4(*args, **kwargs) if bits == 4 else make_step(*args[:6], bits, *args[6:], **kwargs)


def keys_of(s, bits, b, n):
    """float64 [heads, n, d] twice: a sequence's keys, and what bounds the parts that a product with them is made of."""
    if bits == 4:
        return logical4(s.k_pool, s.k_scale, s.table[b], n)
    k = logical(s.k_pool, s.k_scale, s.table[b], n)
    return k, k.abs()


def received(s, bits, b, first=0, causal=True, scale=None, last=0, lse=None):
    """(sums, slack, lse): float64 [key heads, keys], what the keys of sequence b receive from its (last) new tokens, and what fp32 may move of
    it; the rows' log-sum-exps in fp32 (those given, or the reference's own)."""
    n, new, row, group = s.old[b] + s.new[b], s.new[b], int(s.row_start[b]), s.Hq // s.Hkv
    scale = 1.0 / math.sqrt(s.d) if scale is None else scale
    k, k_size = keys_of(s, bits, b, n)
    q = s.q[row:row + new].double().cpu()
    key, pos = torch.arange(n), s.old[b] + torch.arange(new)
    hidden = (key < first)[None, :].expand(new, -1)
    if causal:
        hidden = hidden | (key[None, :] > pos[:, None])
    out, slack = torch.zeros((s.Hkv, n), dtype=torch.float64), torch.zeros((s.Hkv, n), dtype=torch.float64)
    own = torch.zeros((new, s.Hq))
    used = torch.arange(new) >= new - (last or new)
    for h in range(s.Hq):
        g = h // group
        z = q[:, h] @ k[g].T * scale
        own[:, h] = torch.logsumexp(z.masked_fill(hidden, -math.inf), -1).float() if lse is None else lse[row:row + new, h].float().cpu()
        p = torch.exp(z - own[:, h, None].double()).masked_fill(hidden | ~used[:, None], 0.0)
        # a logit is an fp32 sum of at most 132 exact parts (8 bits: of queries in three terms), the log-sum-exp and the difference are rounded
        off = (q[:, h].abs() @ k_size[g].T * scale) * 2.0 ** -15 + own[:, h, None].double().abs() * 2.0 ** -22 + 2.0 ** -20
        out[g] += p.sum(0)
        slack[g] += torch.where(p > 0, p * off, torch.zeros(1, dtype=torch.float64)).sum(0)
    return out, slack + 2.0 ** -20 * out, own


def ledger_of(s, seed, positions=True):
    """Random weights and positions of every place of the pools, on the step's device."""
    gen = torch.Generator().manual_seed(seed)
    shape = s.k_pool.shape[:3]
    weight = torch.exp(2 * torch.randn(shape, generator=gen) - 3)
    position = torch.randint(0, 1 << 20, shape, generator=gen).to(torch.int32)
    return weight.to(s.k_pool.device), position.to(s.k_pool.device) if positions else None


def kept_places(weight, position, keep, n_first, n_recent, n_seen):
    """Places (ascending) that are kept of a sequence's, whose weights and positions these are."""
    def order(i):
        w = float(weight[i])
        always = position[i] < n_first or position[i] >= n_seen - n_recent
        return (not always, 0.0 if always else (math.inf if math.isnan(w) else -w), not always and math.isnan(w), i)
    return sorted(sorted(range(len(weight)), key=order)[:max(min(keep, len(weight)), 0)])


def values_of(bits, pool, scale):
    """float64 values of a whole pool [blocks, heads, tokens, d]."""
    if bits == 4:
        return values(pool, scale)
    if bits == 16:
        return pool.cpu().double()
    return e4m3_values(pool.cpu()) * scale.cpu().double().repeat_interleave(SCALE_TOKENS, -1)[..., None]


__all__ = ["any_step", "kept_places", "keys_of", "ledger_of", "received", "sizes", "values_of"]
