"""Plain 64-bit reference of the cache calls (append with rotation, attention), and steps with shuffled block pools to try them on.
One loop per sequence, everything on the CPU."""
import dataclasses
import math
from typing import List, Optional

import torch

SCALE_TOKENS = 64


def e4m3_values(bytes_):
    return bytes_.view(torch.float8_e4m3fn).to(torch.float32).double()


def pow2_scale(amax: float) -> float:
    """The smallest power of two s >= 2^-100 with amax / s <= 448."""
    if amax == 0:
        return 2.0 ** -100
    e = math.frexp(amax / 448.0)          # m * 2^x, m in [0.5, 1); the quotient by 448 may round, so the power is checked
    s = 2.0 ** (e[1] - 1)
    while amax > 448.0 * s:
        s *= 2.0
    return max(s, 2.0 ** -100)


@dataclasses.dataclass
class Step:
    """A cache with a history, and the new tokens of a step.  Everything is on ``device``."""
    Hq: int
    Hkv: int
    d: int
    block: int
    old: List[int]
    new: List[int]
    rows: int                             # rows of the arrays, some of them behind the last sequence
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    k_scale: Optional[torch.Tensor]
    v_scale: Optional[torch.Tensor]
    table: torch.Tensor
    row_start: torch.Tensor
    seq_lens: torch.Tensor
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor

    def cache(self, spf):
        return spf.KvCache(self.k_pool, self.v_pool, self.k_scale, self.v_scale)

    def step(self, spf, max_new=None):
        return spf.KvStep(self.row_start, self.seq_lens, self.table, max_new or max(max(self.new), 1))


def random_pool(gen, n_blocks, Hkv, block, d, bits, spread=1.0):
    """A pool of N(0, 1) values whose groups of 64 tokens differ in magnitude by powers of two, and its scales."""
    x = torch.randn((n_blocks, Hkv, block // SCALE_TOKENS, SCALE_TOKENS, d), generator=gen)
    x *= 2.0 ** torch.randint(-2, 3, (n_blocks, Hkv, block // SCALE_TOKENS, 1, 1), generator=gen).float() * spread
    if bits == 16:
        return x.view(n_blocks, Hkv, block, d).to(torch.bfloat16), None
    amax = x.abs().amax((-1, -2))
    scale = 2.0 ** torch.ceil(torch.log2(amax / 448.0))
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(n_blocks, Hkv, block, d), scale


def make_step(Hq, Hkv, d, block, old, new, bits, seed=0, behind=0, device="cuda", fused=True):
    """Sequences of old[b] tokens that get new[b] more; pool blocks in random order, some belonging to nobody."""
    gen = torch.Generator().manual_seed(seed)
    lens = [a + b for a, b in zip(old, new)]
    need = [-(-n // block) for n in lens]
    perm = torch.randperm(sum(need) + 2, generator=gen).to(torch.int32)
    table = torch.full((len(old), max(max(need), 1)), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b]) + n]
    k_pool, k_scale = random_pool(gen, sum(need) + 2, Hkv, block, d, bits)
    v_pool, v_scale = random_pool(gen, sum(need) + 2, Hkv, block, d, bits)
    rows = sum(new) + behind
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    qkv = torch.randn((rows, Hq + 2 * Hkv, d), generator=gen).to(torch.bfloat16)
    if not fused:                         # heads outside, as the scoring calls' queries lie
        qkv = qkv.transpose(0, 1).contiguous().transpose(0, 1)
    to = lambda t: None if t is None else t.to(device)  # noqa: E731
    qkv = to(qkv)
    return Step(Hq, Hkv, d, block, list(old), list(new), rows, to(k_pool), to(v_pool), to(k_scale), to(v_scale), to(table),
                to(torch.tensor(starts, dtype=torch.int32)), to(torch.tensor(lens, dtype=torch.int32)), qkv[:, :Hq], qkv[:, Hq:Hq + Hkv],
                qkv[:, Hq + Hkv:])


def rope_table(n, rot_dim, base=10000.0):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * base ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def rotate(x, table, pos, interleaved=False):
    """(rotated, bound): float64 [tokens, heads, d] and a bound on what fp32 with rounded products may be off by."""
    x = x.double().cpu()
    r = table.shape[1]
    c, s = table[pos, :r // 2].double()[:, None], table[pos, r // 2:].double()[:, None]
    part = x[..., :r]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :r // 2], part[..., r // 2:])
    na, nb = a * c - b * s, b * c + a * s
    off = ((a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs())
    out, bound = x.clone(), torch.zeros_like(x)
    for dst, (u, w) in ((out, (na, nb)), (bound, off)):
        if interleaved:
            dst[..., 0:r:2], dst[..., 1:r:2] = u, w
        else:
            dst[..., :r // 2], dst[..., r // 2:r] = u, w
    return out, bound * 2.0 ** -23        # two rounded products and a rounded sum: 2^-24 of each product, 2^-24 of their sum


def logical(pool, scale, table_row, n):
    """float64 [heads, n, d]: a sequence's keys or values in order."""
    ids = table_row[:-(-n // pool.shape[2])].long().cpu() if n else torch.zeros(0, dtype=torch.long)
    x = pool.cpu()[ids]
    if scale is None:
        x = x.double()
    else:
        x = e4m3_values(x) * scale.cpu()[ids].double().repeat_interleave(SCALE_TOKENS, -1)[..., None]
    return x.transpose(0, 1).reshape(pool.shape[1], -1, pool.shape[3])[:, :n]


def attention(q, k, v, pos, first=0, causal=True, scale=None):
    """(out, lse, weight, terms): float64 [rows, heads, d], [rows, heads], sum p |v|, which bounds what a relative error of the
    weights does, and the largest sum |scale q k| of a row's logits, which bounds what fp32 sums do to them; q [rows, Hq, d],
    k and v [Hkv, n, d], pos: the rows' places in the sequence."""
    q = q.double().cpu()
    rows, Hq, d = q.shape
    group = Hq // k.shape[0]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, lse, weight = (torch.zeros((rows, Hq, d), dtype=torch.float64), torch.full((rows, Hq), -math.inf, dtype=torch.float64),
                        torch.zeros((rows, Hq, d), dtype=torch.float64))
    terms = torch.zeros((rows, Hq), dtype=torch.float64)
    for i in range(rows):
        end = min(k.shape[1], int(pos[i]) + 1) if causal else k.shape[1]
        if end <= first:
            continue
        for h in range(Hq):
            kk, vv = k[h // group, first:end], v[h // group, first:end]
            z = kk @ q[i, h] * scale
            lse[i, h] = torch.logsumexp(z, 0)
            p = torch.exp(z - lse[i, h])
            out[i, h] = p @ vv
            weight[i, h] = p @ vv.abs()
            terms[i, h] = (kk.abs() @ q[i, h].abs()).max() * scale
    return out, lse, weight, terms
