"""A draft model's cache in 4 bits, and a cache that is cut to a budget, as cases that can be prepared, run and timed.

A cache in 4 bits holds, for each token and head, its elements as codes 0 ... 15, two to a byte (element 2 j in the low half), and one
bf16 scale for each 32 of them; an element is worth scale * (code - 8).  A ledger beside a cache of any format holds, for each token and
head, the attention weight that it has received and its position.  Four calls work on them:

``append``  rotates a step's queries and keys by their positions and writes keys and values to pools of 4 bits;
``attend``  the attention of a step's tokens over pools of 4 bits (one token a sequence, a few, or a chunk of a prompt);
``weigh``   adds the attention weights of a step's tokens, or of the last ones of it, to the ledger;
``evict``   copies what is kept of sequences to other blocks of the pools: the first tokens, the last ones, and of the others those
            that have received most.

The fields of a case: ``op``; ``bits`` of the cache's elements (4, 8: E4M3 with a scale for 64 tokens, 16: bf16); ``Hq`` query heads,
``Hkv`` key heads, ``d`` head dimension; ``block`` tokens per pool block; ``seqs`` sequences whose new tokens are spread over
[``new_lo``, ``new``] and whose lengths before them over [``old_lo``, ``old``] by ``len_seed`` (the first sequence has the largest of
both); ``last``: the new tokens of a sequence whose weights count (0: all); ``keep``: tokens that are left of a sequence, ``first`` and
``recent`` ones among them in any case.
"""
import math
import random

import numpy as np
import torch

SCALE_TOKENS = 64         # 8 bits: tokens that share a scale
SCALE_DIMS = 32           # 4 bits: elements of a token that share a scale
E4M3_MAX = 448.0
ROPE_BASE = 500000.0
DECAY = 0.96875           # what weights from before a step are multiplied by
own = False               # True: run() makes the calls of the package, False: the operators' plain forms
MAX_DRAWN_PRODUCTS = 1.2e11   # head dimension x heads x rows x keys of a drawn chunk, below the largest listed one's 1.3e11


def _case(name, op, bits, Hq, Hkv, d, block, seqs, new, old, new_lo=None, old_lo=None, len_seed=0, last=0, keep=0, first=0, recent=0):
    return dict(name=name, op=op, bits=bits, Hq=Hq, Hkv=Hkv, d=d, block=block, seqs=seqs, new=new, old=old,
                new_lo=new if new_lo is None else new_lo, old_lo=old if old_lo is None else old_lo, len_seed=len_seed, last=last, keep=keep,
                first=first, recent=recent)


def listed():
    return [
        # one token for each of 32 running sequences: the smallest call, launch latency
        _case("append4_step", "append", 4, 16, 8, 128, 4096, 32, 1, 4095, old_lo=70, len_seed=1),
        # chunks of eight prompts, none of them beginning or ending with a block
        _case("append4_ragged", "append", 4, 16, 8, 128, 4096, 8, 16001, 20000, new_lo=501, old_lo=0, len_seed=2),
        # one lookahead token of one short prompt: latency
        _case("attend4_one", "attend", 4, 32, 8, 64, 4096, 1, 1, 2000),
        # one token for each of 32 running sequences
        _case("attend4_step", "attend", 4, 16, 8, 128, 1024, 32, 1, 16001, old_lo=500, len_seed=3),
        # one token for each of four book-sized prompts: the largest caches
        _case("attend4_long", "attend", 4, 16, 8, 128, 4096, 4, 1, 250003, old_lo=131072, len_seed=5),
        # all eight lookahead tokens at once over a long prompt (the benchmark's draft)
        _case("attend4_lookahead", "attend", 4, 32, 8, 64, 4096, 1, 8, 131072),
        # the last chunk of a prompt of 32k tokens
        _case("attend4_prompt", "attend", 4, 16, 8, 128, 4096, 1, 2048, 30720),
        # the weights of one token of each of 32 running sequences
        _case("weigh_step", "weigh", 4, 16, 8, 128, 1024, 32, 1, 16001, old_lo=500, len_seed=3),
        # the last 32 tokens of a prompt of 32k, as the window that a cut is decided by, bf16
        _case("weigh_window", "weigh", 16, 32, 8, 64, 4096, 1, 2048, 30720, last=32),
        # chunks of three prompts, all of their tokens, over an 8-bit cache, odd lengths
        _case("weigh_prompt", "weigh", 8, 32, 8, 64, 128, 3, 2001, 9001, new_lo=301, old_lo=0, len_seed=6),
        # 32 running sequences that have outgrown a budget of 2048 tokens by some hundred, 4 bits
        _case("evict_running", "evict", 4, 16, 8, 128, 1024, 32, 0, 2500, old_lo=1900, len_seed=7, keep=2048, first=4, recent=256),
        # a prompt of 131072 tokens cut to a quarter, bf16
        _case("evict_prompt", "evict", 16, 16, 8, 128, 4096, 1, 0, 131072, keep=32768, first=4, recent=1024),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))) if hi > lo else lo


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "weigh", "evict"])
    bits = 4 if op in ("append", "attend") else rng.choice([4, 4, 8, 16])
    d = rng.choice([64, 128])
    block = rng.choice([128, 256, 1024, 4096])
    hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 3, 4, 5, 8])
    form = rng.choice(["step", "step", "few", "prompt"])
    new = {"step": 1, "few": rng.randint(2, 16), "prompt": _log(rng, 100, 2048)}[form]
    seqs = rng.choice([1, 1, 2, 3, 8]) if form == "prompt" else _log(rng, 1, 32)
    old = _log(rng, 100, min(131072, 262144 // seqs))
    last = keep = first = recent = 0
    if op == "evict":
        new, keep = 0, max(20, int(old * rng.uniform(0.1, 1.1)))
        first, recent = rng.choice([0, 4, 16]), _log(rng, 1, max(2, keep // 4))
    elif op != "append" and form == "prompt":
        last = rng.choice([0, 16, 64]) if op == "weigh" else 0
        old = min(old, 30000 // seqs)
        while hkv * group * d * seqs * new * (old + new) > MAX_DRAWN_PRODUCTS:
            old, new = old // 2 + 1, new // 2 + 1
    case = _case("", op, bits, hkv * group, hkv, d, block, seqs, new, old, new_lo=max(min(1, new), new // 4), old_lo=old // 4,
                 len_seed=rng.randrange(1 << 20), last=last, keep=keep, first=first, recent=recent)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """(tokens before the step, new tokens) of every sequence."""
    rng = random.Random(case["len_seed"])
    old = [case["old"]] + [rng.randint(case["old_lo"], case["old"]) for _ in range(case["seqs"] - 1)]
    new = [case["new"]] + [rng.randint(case["new_lo"], case["new"]) for _ in range(case["seqs"] - 1)]
    return old, new


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _pow2_scale(amax):
    """8 bits: the smallest power of two s with amax / s <= 448, at least 2^-100."""
    mantissa, exponent = torch.frexp(amax)                            # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875).int()
    return ((torch.where(amax > 0, e, -100).clamp(min=-100) + 127) << 23).view(torch.float32)


def _short_scale(amax):
    """4 bits: the smallest number s of five significant bits with amax / s <= 7, at least 2^-100."""
    s = ((amax / 7.0).view(torch.int32) & -0x80000).view(torch.float32)
    return torch.where(s * 7.0 < amax, (s.view(torch.int32) + 0x80000).view(torch.float32), s).clamp(min=2.0 ** -100)


def _pack4(x):
    """Codes, two to a byte, and scales of fp32 values [..., d]."""
    parts = x.unflatten(-1, (-1, SCALE_DIMS))
    s = _short_scale(parts.abs().amax(-1))
    code = (parts * (1.0 / s)[..., None]).round().clamp(-7, 7).add(8).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), s.to(torch.bfloat16)


def _unpack4(pool, scale):
    """fp32 values of codes and scales."""
    x = torch.stack([pool & 15, pool >> 4], -1).flatten(-2).float().sub_(8.0)
    return x.unflatten(-1, (-1, SCALE_DIMS)).mul_(scale.float()[..., None]).flatten(-2)


def _fill_pools(gen, blocks, heads, tokens, d, bits, size):
    """Keys or values of a cache [blocks, heads, tokens, d] and their scales: channels of different strength, as keys after the
    rotation have, and a slow drift of the magnitude along the tokens."""
    strength = torch.exp(0.5 * _normal(gen, heads, 1, d)) * size
    drift = torch.exp(0.3 * _normal(gen, blocks, heads, tokens // SCALE_TOKENS, 1, 1))
    scale = None
    if bits == 16:
        pool = torch.empty((blocks, heads, tokens, d), dtype=torch.bfloat16, device="cuda")
    elif bits == 8:
        pool = torch.empty((blocks, heads, tokens, d), dtype=torch.uint8, device="cuda")
        scale = torch.empty((blocks, heads, tokens // SCALE_TOKENS), dtype=torch.float32, device="cuda")
    else:
        pool = torch.empty((blocks, heads, tokens, d // 2), dtype=torch.uint8, device="cuda")
        scale = torch.empty((blocks, heads, tokens, d // SCALE_DIMS), dtype=torch.bfloat16, device="cuda")
    at_once = max(1, (1 << 25) // (heads * tokens * d))
    for i in range(0, blocks, at_once):
        n = min(at_once, blocks - i)
        x = (_normal(gen, n, heads, tokens, d) * strength).unflatten(2, (-1, SCALE_TOKENS)) * drift[i:i + n]
        if bits == 16:
            pool[i:i + n] = x.flatten(2, 3).to(torch.bfloat16)
        elif bits == 8:
            s = _pow2_scale(x.abs().amax((-1, -2)))
            scale[i:i + n] = s
            pool[i:i + n] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).flatten(2, 3)
        else:
            pool[i:i + n], scale[i:i + n] = _pack4(x.flatten(2, 3))
    return pool, scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 17)
    op, Hq, Hkv, d, block = (case[x] for x in ("op", "Hq", "Hkv", "d", "block"))
    i32 = dict(dtype=torch.int32, device="cuda")
    old, new = _lengths(case)
    lens = [a + b for a, b in zip(old, new)]
    need = [-(-x // block) for x in lens]
    to_need = -(-case["keep"] // block) if op == "evict" else 0        # blocks that a sequence is copied to
    blocks = sum(need) + case["seqs"] * to_need + 2
    perm = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["seqs"], max(need)), -1, **i32)
    for b, k in enumerate(need):
        table[b, :k] = perm[sum(need[:b]):sum(need[:b]) + k]
    k_pool, k_scale = _fill_pools(gen, blocks, Hkv, block, d, case["bits"], 1.0)
    v_pool, v_scale = _fill_pools(gen, blocks, Hkv, block, d, case["bits"], 0.7)
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    rows = starts[-1]
    state = dict(case=case, k_pool=k_pool, v_pool=v_pool, k_scale=k_scale, v_scale=v_scale, block_table=table,
                 row_start=torch.tensor(starts, **i32), seq_lens=torch.tensor(lens, **i32), rows=rows, max_new=max(new), max_len=max(lens),
                 status=torch.zeros(1, **i32), workspace=None)
    if op == "append":
        # the fused projection's output: queries, keys and values of a token side by side
        qkv = _normal(gen, rows, Hq + 2 * Hkv, d) * torch.exp(0.5 * _normal(gen, Hq + 2 * Hkv, d))
        qkv = qkv.to(torch.bfloat16)
        inv = ROPE_BASE ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        angle = torch.arange(max(lens), device="cuda", dtype=torch.float64)[:, None] * inv
        state.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], rope=torch.cat([angle.cos(), angle.sin()], 1).float(),
                     q_out=torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda"))
        return state
    if op in ("attend", "weigh"):
        q = _normal(gen, rows, Hq, d) * 1.5
        state.update(q=q.to(torch.bfloat16), out=torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda"),
                     lse=torch.zeros((rows, Hq), dtype=torch.float32, device="cuda"))
    if op == "weigh":
        # what the step's attention has left: the log-sum-exps of its rows
        z, row, live = _logits(state)
        state["lse"][row[live]] = torch.logsumexp(z, -1).permute(0, 3, 1, 2).flatten(2)[live]
        del z
        seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), state["row_start"].diff().long())
        before = torch.randint(0, 5000, (case["seqs"],), generator=gen, device="cuda")   # tokens that were evicted earlier
        place = torch.arange(rows, device="cuda") - state["row_start"].long()[seq] + (state["seq_lens"] - state["row_start"].diff()).long()[seq]
        state["positions"] = (place + before[seq]).to(torch.int32)
    if op in ("weigh", "evict"):
        # received weights are spread over some orders of magnitude; positions rise along a sequence, with gaps of earlier cuts
        weight = torch.exp(2.5 * _normal(gen, blocks, Hkv, block) - 6.0)
        state.update(weight=weight, position=torch.zeros((blocks, Hkv, block), **i32))
    if op == "evict":
        gaps = torch.randint(0, 3, (case["seqs"], Hkv, max(need) * block), generator=gen, device="cuda")
        position = (gaps.cumsum(-1) // 2 + torch.arange(max(need) * block, device="cuda")).to(torch.int32)
        for b, k in enumerate(need):
            state["position"][table[b, :k].long()] = position[b, :, :k * block].unflatten(-1, (k, block)).transpose(0, 1)
        last = torch.stack([position[b, :, max(n - 1, 0)].max() for b, n in enumerate(lens)])
        to_table = perm[sum(need):sum(need) + case["seqs"] * to_need].view(case["seqs"], to_need)
        state.update(to_table=to_table.contiguous(), to_lens=torch.zeros(case["seqs"], **i32), keep=torch.full((case["seqs"],), case["keep"], **i32),
                     n_seen=(last + 1).to(torch.int32))
    return state


# ---------------------------------------------------------------------------------------------- the calls
def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "weigh": _own_weigh, "evict": _own_evict}[op](state)
    return {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}[op](state)


def _own_cache(spf, state):
    return spf.KvCache(state["k_pool"], state["v_pool"], state["k_scale"], state["v_scale"])


def _own_step(spf, state):
    return spf.KvStep(state["row_start"], state["seq_lens"], state["block_table"], state["max_new"])


def _pools(state):
    """What a cache holds: bf16, E4M3 values and their scales, or codes, two to a byte, and their scales."""
    if state["case"]["bits"] == 16:
        return dict(k=state["k_pool"], v=state["v_pool"])
    held = torch.float8_e4m3fn if state["case"]["bits"] == 8 else torch.uint8
    return dict(k=state["k_pool"].view(held), v=state["v_pool"].view(held), k_scale=state["k_scale"], v_scale=state["v_scale"])


def _own_append(state):
    import paper_2603_02631_b200 as spf
    spf.spf_kv_append(_own_cache(spf, state), _own_step(spf, state), state["k"], state["v"], q=state["q"], q_out=state["q_out"],
                      rope=spf.Rope(state["rope"]), dev_status=state["status"])
    return dict(q=state["q_out"], **_pools(state))


def _own_attend(state):
    import paper_2603_02631_b200 as spf
    cache, step = _own_cache(spf, state), _own_step(spf, state)
    if state["workspace"] is None:
        state["workspace"] = torch.empty(spf.spf_attend_workspace_bytes(cache, step, state["q"]), dtype=torch.uint8, device="cuda")
    spf.spf_attend(cache, step, state["q"], state["out"], state["workspace"], lse=state["lse"], dev_status=state["status"])
    return dict(out=state["out"], lse=state["lse"])


def _own_weigh(state):
    import paper_2603_02631_b200 as spf
    spf.spf_kv_weigh(_own_cache(spf, state), _own_step(spf, state), state["q"], state["lse"], spf.KvLedger(state["weight"], state["position"]),
                     positions=state["positions"], last_rows=state["case"]["last"], decay=DECAY, dev_status=state["status"])
    return dict(weight=state["weight"], position=state["position"])


def _own_evict(state):
    import paper_2603_02631_b200 as spf
    cache = _own_cache(spf, state)
    if state["workspace"] is None:
        state["workspace"] = torch.empty(spf.spf_kv_evict_workspace_bytes(cache, state["to_table"]), dtype=torch.uint8, device="cuda")
    spf.spf_kv_evict(cache, spf.KvLedger(state["weight"], state["position"]), state["seq_lens"], state["block_table"], state["keep"],
                     state["to_table"], state["to_lens"], state["workspace"], n_first=state["case"]["first"], n_recent=state["case"]["recent"],
                     n_seen=state["n_seen"], dev_status=state["status"])
    return dict(lens=state["to_lens"], weight=state["weight"], position=state["position"], **_pools(state))


# ---------------------------------------------------------------------------------------------- plain forms
def _rows(state):
    """(sequence, position) of every row of the step."""
    row = torch.arange(state["rows"], device="cuda")
    start = state["row_start"].long()
    seq = torch.searchsorted(start, row, right=True) - 1
    return seq, state["seq_lens"].long()[seq] - (start[seq + 1] - row)


def _rotate(x, table, pos):
    x, half = x.float(), x.shape[-1] // 2
    cos, sin = table[pos, None, :half], table[pos, None, half:]
    return torch.cat([x[..., :half] * cos - x[..., half:] * sin, x[..., half:] * cos + x[..., :half] * sin], -1)


def _plain_append(state):
    seq, pos = _rows(state)
    block = state["case"]["block"]
    at, off = state["block_table"][seq, pos // block].long(), pos % block
    state["q_out"].copy_(_rotate(state["q"], state["rope"], pos).to(torch.bfloat16))
    state["k_pool"][at, :, off], state["k_scale"][at, :, off] = _pack4(_rotate(state["k"], state["rope"], pos))
    state["v_pool"][at, :, off], state["v_scale"][at, :, off] = _pack4(state["v"].float())
    return dict(q=state["q_out"], **_pools(state))


def _gathered(pool, scale, bits, table, length):
    """fp32 [sequences, heads, length, d] of a paged cache; what a table's unused entries point to is masked later."""
    ids = table.clamp(min=0).long()
    if bits == 16:
        x = pool[ids].float()                                          # [seqs, blocks, heads, tokens, d]
    elif bits == 8:
        x = pool[ids].view(torch.float8_e4m3fn).float()
        x = x.unflatten(3, (-1, SCALE_TOKENS)).mul_(scale[ids][..., None, None]).flatten(3, 4)
    else:
        x = _unpack4(pool[ids], scale[ids])
    return x.transpose(1, 2).flatten(2, 3)[:, :, :length]


def _logits(state):
    """fp32 logits [sequences, key heads, group, new, keys] of the sequences' (last) new tokens, -inf where a row does not see a key, the
    rows of [sequences, new] in the step's arrays, and which of them exist."""
    case = state["case"]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    B, new = case["seqs"], min(state["max_new"], case["last"] or state["max_new"])
    k = _gathered(state["k_pool"], state["k_scale"], case["bits"], state["block_table"], state["max_len"])
    start, count = state["row_start"][:-1].long(), state["row_start"].diff().long()
    i = count[:, None] - new + torch.arange(new, device="cuda")        # [seqs, new]; below zero: dropped later
    row = start[:, None] + i.clamp(min=0)
    q = state["q"][row].float().view(B, new, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    last = (state["seq_lens"].long() - count)[:, None] + i             # the position of a row, the last key that it sees
    z = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(B, Hkv, Hq // Hkv, new, -1)
    z.masked_fill_(torch.arange(k.shape[2], device="cuda") > last[:, None, None, :, None], float("-inf"))
    return z, row, i >= 0


def _plain_attend(state):
    B, new, Hq, d = state["case"]["seqs"], state["max_new"], state["case"]["Hq"], state["case"]["d"]
    z, row, live = _logits(state)
    v = _gathered(state["v_pool"], state["v_scale"], state["case"]["bits"], state["block_table"], state["max_len"])
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    # a sequence's own length hides what a shorter one has behind it; its values there are finite, so a zero weight is enough
    o = (p.flatten(2, 3) @ v).view(*p.shape[:-1], d) / total
    lse = (top + total.log())[..., 0]
    state["out"][row[live]] = o.permute(0, 3, 1, 2, 4).reshape(B, new, Hq, d)[live].to(torch.bfloat16)
    state["lse"][row[live]] = lse.permute(0, 3, 1, 2).reshape(B, new, Hq)[live]
    return dict(out=state["out"], lse=state["lse"])


def _plain_weigh(state):
    case = state["case"]
    B, Hkv, block = case["seqs"], case["Hkv"], case["block"]
    z, row, live = _logits(state)
    count = state["row_start"].diff().long()
    lse = state["lse"][row].unflatten(-1, (Hkv, -1)).permute(0, 2, 3, 1)[..., None]
    p = z.sub_(lse).exp_().masked_fill_(~live[:, None, None, :, None], 0.0)
    got = p.sum((2, 3))                                                # [seqs, Hkv, keys]
    seq, key = torch.nonzero(torch.arange(state["max_len"], device="cuda") < state["seq_lens"][:, None], as_tuple=True)
    at, off = state["block_table"][seq, key // block].long(), key % block
    fresh = key >= (state["seq_lens"].long() - count)[seq]
    before = state["weight"][at, :, off] * DECAY
    state["weight"][at, :, off] = torch.where(fresh[:, None], torch.zeros_like(before), before) + got[seq, :, key]
    seq, pos = _rows(state)
    state["position"][state["block_table"][seq, pos // block].long(), :, pos % block] = state["positions"][:, None].expand(-1, Hkv)
    return dict(weight=state["weight"], position=state["position"])


def _plain_evict(state):
    case = state["case"]
    block, bits = case["block"], case["bits"]
    lens, n = state["seq_lens"].long(), state["max_len"]
    ids = state["block_table"].clamp(min=0).long()
    place = torch.arange(n, device="cuda")
    weight = state["weight"][ids].transpose(1, 2).flatten(2)[:, :, :n]
    position = state["position"][ids].transpose(1, 2).flatten(2)[:, :, :n]
    always = (position < case["first"]) | (position >= (state["n_seen"] - case["recent"])[:, None, None])
    weight = weight.masked_fill(always, float("inf")).masked_fill_(place >= lens[:, None, None], float("-inf"))
    order = weight.sort(dim=-1, descending=True, stable=True).indices
    left = torch.minimum(lens, state["keep"].long())
    kept = torch.zeros_like(weight, dtype=torch.bool).scatter_(-1, order, (place < left[:, None, None]).expand_as(order))
    seq, head, key = torch.nonzero(kept, as_tuple=True)                # in order of the places
    to = (kept.cumsum(-1) - 1)[seq, head, key]
    src, dst = state["block_table"][seq, key // block].long(), state["to_table"][seq, to // block].long()
    key, to = key % block, to % block
    state["weight"][dst, head, to] = state["weight"][src, head, key]
    state["position"][dst, head, to] = state["position"][src, head, key]
    if bits == 8:
        _move8(state["k_pool"], state["k_scale"], src, dst, head, key, to)
        _move8(state["v_pool"], state["v_scale"], src, dst, head, key, to)
    else:
        state["k_pool"][dst, head, to] = state["k_pool"][src, head, key]
        state["v_pool"][dst, head, to] = state["v_pool"][src, head, key]
        if bits == 4:
            state["k_scale"][dst, head, to] = state["k_scale"][src, head, key]
            state["v_scale"][dst, head, to] = state["v_scale"][src, head, key]
    state["to_lens"].copy_(left)
    return dict(lens=state["to_lens"], weight=state["weight"], position=state["position"], **_pools(state))


def _move8(pool, scale, src, dst, head, key, to):
    """8 bits: a group's scale becomes the largest of its tokens', whose bytes are rounded to it."""
    was = scale[src, head, key // SCALE_TOKENS]
    cell = (dst * scale.shape[1] + head) * scale.shape[2] + to // SCALE_TOKENS
    now = torch.zeros_like(scale).view(-1).scatter_reduce_(0, cell, was, "amax")[cell]
    x = pool[src, head, key].view(torch.float8_e4m3fn).float() * (was / now)[:, None]
    pool[dst, head, to] = x.to(torch.float8_e4m3fn).view(torch.uint8)
    scale.view(-1)[cell] = now


# ---------------------------------------------------------------------------------------------- 64 bits
def _wide(s, name, ids, head):
    """float64 [tokens, d] of some blocks of a head."""
    pool, bits = s[name + "_pool"][ids, head], s["case"]["bits"]
    if bits == 16:
        return pool.double().flatten(0, 1)
    scale = s[name + "_scale"][ids, head].double()
    if bits == 8:
        return (pool.view(torch.float8_e4m3fn).to(torch.float32).double() * scale.repeat_interleave(SCALE_TOKENS, -1)[..., None]).flatten(0, 1)
    x = torch.empty((*pool.shape[:-1], s["case"]["d"]), dtype=torch.float64, device="cuda")
    x[..., 0::2], x[..., 1::2] = (pool % 16).double() - 8, (pool // 16).double() - 8
    return (x * scale.repeat_interleave(SCALE_DIMS, -1)).flatten(0, 1)


def exact(case, seed):
    s = prepare(case, seed)
    old, new = _lengths(case)
    return {"append": _exact_append, "attend": _exact_attend, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](case, s, old, new)


def _exact_attend(case, s, old, new):
    d, group, block = case["d"], case["Hq"] // case["Hkv"], case["block"]
    out, lse = torch.zeros_like(s["out"], dtype=torch.float64), torch.zeros_like(s["lse"], dtype=torch.float64)
    row = 0
    for b, (before, count) in enumerate(zip(old, new)):
        ids = s["block_table"][b, :-(-(before + count) // block)].long()
        hidden = torch.arange(before + count, device="cuda")[None, :] > (before + torch.arange(count, device="cuda"))[:, None]
        for h in range(case["Hkv"]):
            k, v = (_wide(s, x, ids, h)[:before + count] for x in "kv")
            for g in range(h * group, (h + 1) * group):
                z = s["q"][row:row + count, g].double() @ k.T / math.sqrt(d)
                z[hidden] = -math.inf
                lse[row:row + count, g] = torch.logsumexp(z, -1)
                out[row:row + count, g] = torch.exp(z - lse[row:row + count, g, None]) @ v
        row += count
    return dict(out=out, lse=lse)


def _exact_weigh(case, s, old, new):
    group, block = case["Hq"] // case["Hkv"], case["block"]
    weight, position = s["weight"].double(), s["position"].clone()
    row = 0
    for b, (before, count) in enumerate(zip(old, new)):
        n = before + count
        ids = s["block_table"][b, :-(-n // block)].long()
        used = min(count, case["last"]) if case["last"] else count
        i = torch.arange(count - used, count, device="cuda")
        hidden = torch.arange(n, device="cuda")[None, :] > (before + i)[:, None]
        place = torch.arange(n, device="cuda")
        for h in range(case["Hkv"]):
            k = _wide(s, "k", ids, h)[:n]
            got = torch.zeros(n, dtype=torch.float64, device="cuda")
            for g in range(h * group, (h + 1) * group):
                z = s["q"][row + i, g].double() @ k.T / math.sqrt(case["d"]) - s["lse"][row + i, g].double()[:, None]
                got += torch.exp(z).masked_fill_(hidden, 0.0).sum(0)
            at = ids[place // block], h, place % block
            weight[at] = torch.where(place < before, weight[at] * DECAY, 0.0) + got
            position[at[0][before:], h, at[2][before:]] = s["positions"][row:row + count]
        row += count
    return dict(weight=weight, position=position)


def _exact_evict(case, s, old, new):
    block, bits = case["block"], case["bits"]
    lens = torch.tensor([min(n, case["keep"]) for n in old], dtype=torch.int32, device="cuda")
    got = {"k": s["k_pool"].clone(), "v": s["v_pool"].clone()}
    if bits == 16:
        got = {x: got[x].double() for x in got}
    if bits == 8:
        got = {x: got[x].view(torch.float8_e4m3fn).to(torch.float32).double() for x in got}
    if bits != 16:
        got |= {x: s[x].double() for x in ("k_scale", "v_scale")}
    weight, position = s["weight"].double(), s["position"].clone()
    for b, n in enumerate(old):
        src, dst = (s[x][b].long().cpu().numpy() for x in ("block_table", "to_table"))
        place = np.arange(n)
        for h in range(case["Hkv"]):
            at = (torch.from_numpy(src[place // block]).cuda(), h, torch.from_numpy(place % block).cuda())
            w, p = s["weight"][at].double().cpu().numpy(), s["position"][at].cpu().numpy()
            always = (p < case["first"]) | (p >= int(s["n_seen"][b]) - case["recent"])
            ranked = np.lexsort((place, -w, ~always))                  # the last key is the first that counts
            kept = np.sort(ranked[:min(n, case["keep"])])
            to = np.arange(len(kept))
            source = (torch.from_numpy(src[kept // block]).cuda(), h, torch.from_numpy(kept % block).cuda())
            place_to = (torch.from_numpy(dst[to // block]).cuda(), h, torch.from_numpy(to % block).cuda())
            weight[place_to], position[place_to] = s["weight"][source].double(), s["position"][source]
            for x in "kv":
                if bits != 8:
                    got[x][place_to] = s[x + "_pool"][source].to(got[x].dtype)
                    if bits == 4:
                        got[x + "_scale"][place_to] = s[x + "_scale"][source].double()
                    continue
                was = s[x + "_scale"][source[0], h, source[2] // SCALE_TOKENS].double()
                bytes_ = s[x + "_pool"][source].view(torch.float8_e4m3fn).to(torch.float32).double()
                padded = torch.zeros(-(-len(kept) // SCALE_TOKENS) * SCALE_TOKENS, dtype=torch.float64, device="cuda")
                padded[:len(kept)] = was
                now = padded.view(-1, SCALE_TOKENS).amax(1).repeat_interleave(SCALE_TOKENS)[:len(kept)]
                got[x][place_to] = bytes_ * (was / now)[:, None]
                got[x + "_scale"][place_to[0], h, place_to[2] // SCALE_TOKENS] = now
    return dict(lens=lens, weight=weight, position=position, **got)


def _exact_append(case, s, old, new):
    """Rotated queries and the scales; a code, which is the nearest whole number, has no value between two."""
    d, block, half = case["d"], case["block"], case["d"] // 2
    # all numbers of five significant bits that a scale can be
    powers = torch.tensor([2.0 ** e * (16 + m) for e in range(-104, 122) for m in range(16)], dtype=torch.float64, device="cuda")
    got = dict(q=torch.zeros_like(s["q_out"], dtype=torch.float64), k=None, v=None, k_scale=s["k_scale"].double(), v_scale=s["v_scale"].double())
    row = 0
    for b, (before, count) in enumerate(zip(old, new)):
        pos = torch.arange(before, before + count, device="cuda")
        at, off = s["block_table"][b].long()[pos // block], pos % block
        cos, sin = s["rope"][pos, :half].double()[:, None], s["rope"][pos, half:].double()[:, None]
        turned = {"v": s["v"][row:row + count].double()}
        for x in "qk":
            a = s[x][row:row + count].double()
            turned[x] = torch.cat([a[..., :half] * cos - a[..., half:] * sin, a[..., half:] * cos + a[..., :half] * sin], -1)
        got["q"][row:row + count] = turned["q"]
        for x in "kv":
            top = turned[x].reshape(count, case["Hkv"], -1, SCALE_DIMS).abs().amax(-1)
            got[x + "_scale"][at, :, off] = powers[torch.searchsorted(powers * 7, top)]
        row += count
    return got


# ---------------------------------------------------------------------------------------------- floors
def _token_bytes(case):
    """Bytes of a token's key, or value, of one head."""
    return {16: 2 * case["d"], 8: case["d"] + 4 / SCALE_TOKENS, 4: case["d"] / 2 + 2 * case["d"] / SCALE_DIMS}[case["bits"]]


def work(case):
    """Each input read once, each output written once: of cache and ledger, the rows that the call is about."""
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    old, new = _lengths(case)
    rows, size = sum(new), _token_bytes(case)
    if case["op"] == "append":
        return {"bytes": rows * (4 * Hq * d + 2 * Hkv * (2 * d + size)) + 4 * d * max(a + b for a, b in zip(old, new)), "flops": 3.0 * rows * d * (Hq + Hkv)}
    if case["op"] == "evict":
        left = sum(min(n, case["keep"]) for n in old)
        return {"bytes": Hkv * (8 * sum(old) + left * (2 * 2 * size + 2 * 8)), "flops": 0.0}
    keys = sum(a + b for a, b in zip(old, new))
    if case["op"] == "attend":
        pairs = sum(b * a + b * (b + 1) // 2 for a, b in zip(old, new))
        return {"bytes": 2 * Hkv * keys * size + rows * Hq * (4 * d + 4), "flops": 4.0 * Hq * d * pairs}
    used = [min(b, case["last"]) if case["last"] else b for b in new]
    pairs = sum(u * (a + b - u) + u * (u + 1) // 2 for a, b, u in zip(old, new, used))
    return {"bytes": Hkv * (keys * (size + 8) + rows * 4) + sum(used) * Hq * (2 * d + 4), "flops": 2.0 * Hq * d * pairs}
