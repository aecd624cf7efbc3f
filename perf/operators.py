"""The draft model's cache operators, as cases that can be prepared, run and timed.

A draft model that is served beside the scoring calls keeps its keys and values in block pools, in bf16 or in 8 bits (E4M3
with one scale for each 64 tokens of a block and head).  Three calls work on them:

``append``  rotates a step's queries and keys by their positions and writes keys and values to the pools;
``attend``  the attention of a step's tokens over the pools (one token a sequence, a few, or a chunk of a prompt);
``score``   the token importance of a prompt whose keys are in 8-bit pools.

The fields of a case: ``op``; ``bits`` of the cache's elements (16: bf16, 8); ``Hq`` query heads, ``Hkv`` key heads, ``d``
head dimension; ``block`` tokens per pool block; ``seqs`` sequences whose new tokens are spread over [``new_lo``, ``new``] and
whose lengths before them over [``old_lo``, ``old``] by ``len_seed`` (the first sequence has the largest of both); for scoring
``L`` layers, ``m`` lookahead queries and ``n`` prompt tokens.
"""
import math
import random

import torch

SCALE_TOKENS = 64         # tokens that share a scale in an 8-bit pool
E4M3_MAX = 448.0
ROPE_BASE = 500000.0
own = False               # True: run() makes the calls of the package, False: the operators' plain forms
MAX_DRAWN_PRODUCTS = 1.2e11   # head dimension x heads x rows x keys of a drawn chunk, below the largest listed one's 1.3e11


def _case(name, op, bits, Hq, Hkv, d, block, seqs, new, old, new_lo=None, old_lo=None, len_seed=0):
    return dict(name=name, op=op, bits=bits, Hq=Hq, Hkv=Hkv, d=d, block=block, seqs=seqs, new=new, old=old,
                new_lo=new if new_lo is None else new_lo, old_lo=old if old_lo is None else old_lo, len_seed=len_seed)


def _score(name, L, Hq, Hkv, d, m, n, block):
    return dict(name=name, op="score", bits=8, L=L, Hq=Hq, Hkv=Hkv, d=d, m=m, n=n, block=block)


def listed():
    return [
        # one token for each of 32 running sequences, into an 8-bit cache: the smallest call, launch latency
        _case("append_step_fp8", "append", 8, 16, 8, 128, 4096, 32, 1, 4095, old_lo=70, len_seed=1),
        # a whole prompt of 8k tokens into a bf16 cache (16-layer draft with heads of 64)
        _case("append_prompt", "append", 16, 32, 8, 64, 4096, 1, 8192, 0),
        # chunks of eight prompts into an 8-bit cache, none of them beginning or ending with a block
        _case("append_ragged_fp8", "append", 8, 16, 8, 128, 4096, 8, 16001, 20000, new_lo=501, old_lo=0, len_seed=2),
        # one lookahead token of one short prompt: latency
        _case("attend_one", "attend", 16, 32, 8, 64, 4096, 1, 1, 2000),
        # one token for each of 32 running sequences over an 8-bit cache
        _case("attend_step_fp8", "attend", 8, 16, 8, 128, 1024, 32, 1, 16001, old_lo=500, len_seed=3),
        # one token for each of 16 running sequences of 4 to 32k tokens over a bf16 cache
        _case("attend_step", "attend", 16, 16, 8, 128, 256, 16, 1, 32767, old_lo=4001, len_seed=4),
        # all eight lookahead tokens at once over a long prompt (the benchmark's draft)
        _case("attend_lookahead", "attend", 16, 32, 8, 64, 4096, 1, 8, 131072),
        # one token for each of four book-sized prompts, 8 bits: the largest caches
        _case("attend_long_fp8", "attend", 8, 16, 8, 128, 4096, 4, 1, 250003, old_lo=131072, len_seed=5),
        # the last chunk of a prompt of 32k tokens
        _case("attend_prompt", "attend", 16, 16, 8, 128, 4096, 1, 2048, 30720),
        # chunks of four prompts over an 8-bit cache, odd lengths
        _case("attend_prompt_fp8", "attend", 8, 32, 8, 64, 128, 4, 2001, 9001, new_lo=301, old_lo=0, len_seed=6),
        # the importance of a chat-length prompt's tokens from an 8-bit cache with the smallest blocks
        _score("score_4k_fp8", 16, 32, 8, 64, 8, 4001, 128),
        # and of the benchmark's long context
        _score("score_128k_fp8", 16, 32, 8, 64, 16, 131072, 4096),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))) if hi > lo else lo


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "score"])
    d = rng.choice([64, 128])
    block = rng.choice([128, 256, 1024, 4096])
    hkv = rng.choice([1, 2, 4, 8, 8])
    group = rng.choice([1, 2, 3, 4, 5, 8])
    if op == "score":
        m = rng.choice([1, 4, 5, 8, 8, 16])
        group = rng.choice([g for g in (1, 2, 3, 4, 8) if g * (-(-m // 8) * 8) <= 64])
        case = _score("", rng.choice([2, 4, 12, 16]), hkv * group, hkv, d, m, _log(rng, 500, 65536), block)
    else:
        form = rng.choice(["step", "step", "few", "prompt"])
        new = {"step": 1, "few": rng.randint(2, 16), "prompt": _log(rng, 100, 2048)}[form]
        seqs = rng.choice([1, 1, 2, 3, 8]) if form == "prompt" else _log(rng, 1, 32)
        old = _log(rng, 100, min(131072, 262144 // seqs))
        if op == "attend" and form == "prompt":
            old = min(old, 30000 // seqs)
            while hkv * group * d * seqs * new * (old + new) > MAX_DRAWN_PRODUCTS:
                old, new = old // 2 + 1, new // 2 + 1
        case = _case("", op, rng.choice([8, 8, 16]), hkv * group, hkv, d, block, seqs, new, old, new_lo=max(1, new // 4),
                     old_lo=old // 4, len_seed=rng.randrange(1 << 20))
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
    """The smallest power of two s with amax / s <= 448, at least 2^-100."""
    mantissa, exponent = torch.frexp(amax)                            # amax = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875).int()
    return ((torch.where(amax > 0, e, -100).clamp(min=-100) + 127) << 23).view(torch.float32)


def _fill_pools(gen, shape, bits, queries_like):
    """Keys or values of a cache as bf16 pools [..., blocks, heads, tokens, d], or as 8-bit pools with their scales: channels of
    different strength, as keys after the rotation have, and a slow drift of the magnitude along the tokens."""
    *lead, tokens, d = shape
    heads = lead[-1]
    strength = torch.exp(0.5 * _normal(gen, heads, 1, d)) * queries_like
    drift = torch.exp(0.3 * _normal(gen, *lead, tokens // SCALE_TOKENS, 1, 1))
    pool = torch.empty(shape, dtype=torch.bfloat16 if bits == 16 else torch.uint8, device="cuda")
    scale = torch.empty(tuple(lead) + (tokens // SCALE_TOKENS,), dtype=torch.float32, device="cuda") if bits == 8 else None
    for i in range(shape[0]):
        x = _normal(gen, *shape[1:]) * strength
        x = x.view(*shape[1:-2], tokens // SCALE_TOKENS, SCALE_TOKENS, d) * drift[i]
        if bits == 16:
            pool[i] = x.view(shape[1:]).to(torch.bfloat16)
        else:
            s = _pow2_scale(x.abs().amax((-1, -2)))
            scale[i] = s
            pool[i] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(shape[1:])
    return pool, scale


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * seed + 17)
    Hq, Hkv, d, block = (case[x] for x in ("Hq", "Hkv", "d", "block"))
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["op"] == "score":
        L, m, n = case["L"], case["m"], case["n"]
        blocks = -(-n // block)
        pool, scale = _fill_pools(gen, (L, blocks + 1, Hkv, block, d), 8, 1.0)
        q = _normal(gen, L, Hq, m, d)
        # spans of keys that a quarter of the heads look for: what the importance is there to find
        spans = torch.randint(0, blocks * block // 64, (16,), generator=gen, device="cuda")
        table = torch.randperm(blocks + 1, generator=gen, device="cuda")[:blocks]
        for l in range(0, L, 4):
            at = table[spans * 64 // block], (spans * 64 % block)
            for k in range(16):
                pool[l, at[0][k], 0, at[1][k] + torch.arange(16, device="cuda")] = \
                    (q[l, 0, 0] * 96).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        return dict(case=case, q=q.to(torch.bfloat16), k_pools=list(pool.unbind(0)), k_scales=list(scale.unbind(0)), pool=pool, scale=scale,
                    block_table=table.to(torch.int32), importance=torch.zeros(n, dtype=torch.float32, device="cuda"),
                    lse=torch.zeros((L, Hq, m), dtype=torch.float32, device="cuda"), status=torch.zeros(1, **i32), workspace=None)
    old, new = _lengths(case)
    lens = [a + b for a, b in zip(old, new)]
    need = [-(-x // block) for x in lens]
    perm = torch.randperm(sum(need) + 2, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["seqs"], max(need)), -1, **i32)
    for b, k in enumerate(need):
        table[b, :k] = perm[sum(need[:b]):sum(need[:b]) + k]
    k_pool, k_scale = _fill_pools(gen, (sum(need) + 2, Hkv, block, d), case["bits"], 1.0)
    v_pool, v_scale = _fill_pools(gen, (sum(need) + 2, Hkv, block, d), case["bits"], 0.7)
    starts = [sum(new[:b]) for b in range(len(new) + 1)]
    rows = starts[-1]
    state = dict(case=case, k_pool=k_pool, v_pool=v_pool, k_scale=k_scale, v_scale=v_scale, block_table=table,
                 row_start=torch.tensor(starts, **i32), seq_lens=torch.tensor(lens, **i32), rows=rows, max_new=max(new), max_len=max(lens),
                 status=torch.zeros(1, **i32), workspace=None)
    if case["op"] == "append":
        # the fused projection's output: queries, keys and values of a token side by side
        qkv = _normal(gen, rows, Hq + 2 * Hkv, d) * torch.exp(0.5 * _normal(gen, Hq + 2 * Hkv, d))
        qkv = qkv.to(torch.bfloat16)
        inv = ROPE_BASE ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        angle = torch.arange(max(lens), device="cuda", dtype=torch.float64)[:, None] * inv
        state.update(q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:], rope=torch.cat([angle.cos(), angle.sin()], 1).float(),
                     q_out=torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda"))
    else:
        q = _normal(gen, rows, Hq, d) * 1.5
        state.update(q=q.to(torch.bfloat16), out=torch.zeros((rows, Hq, d), dtype=torch.bfloat16, device="cuda"),
                     lse=torch.zeros((rows, Hq), dtype=torch.float32, device="cuda"))
    return state


# ---------------------------------------------------------------------------------------------- the calls
def run(state):
    op = state["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "score": _own_score}[op](state)
    return {"append": _plain_append, "attend": _plain_attend, "score": _plain_score}[op](state)


def _own_cache(spf, state):
    return (spf.KvCache(state["k_pool"], state["v_pool"], state["k_scale"], state["v_scale"]),
            spf.KvStep(state["row_start"], state["seq_lens"], state["block_table"], state["max_new"]))


def _appended(state):
    if state["case"]["bits"] == 16:
        return dict(q=state["q_out"], k=state["k_pool"], v=state["v_pool"])
    return dict(q=state["q_out"], k=state["k_pool"].view(torch.float8_e4m3fn), v=state["v_pool"].view(torch.float8_e4m3fn),
                k_scale=state["k_scale"], v_scale=state["v_scale"])


def _own_append(state):
    import paper_2603_02631_b200 as spf
    cache, step = _own_cache(spf, state)
    spf.spf_kv_append(cache, step, state["k"], state["v"], q=state["q"], q_out=state["q_out"], rope=spf.Rope(state["rope"]),
                      dev_status=state["status"])
    return _appended(state)


def _own_attend(state):
    import paper_2603_02631_b200 as spf
    cache, step = _own_cache(spf, state)
    if state["workspace"] is None:
        state["workspace"] = torch.empty(spf.spf_attend_workspace_bytes(cache, step, state["q"]), dtype=torch.uint8, device="cuda")
    spf.spf_attend(cache, step, state["q"], state["out"], state["workspace"], lse=state["lse"], dev_status=state["status"])
    return dict(out=state["out"], lse=state["lse"])


def _own_score(state):
    import paper_2603_02631_b200 as spf
    prompt = spf.PagedFp8PromptBuffers(state["q"], state["k_pools"], state["k_scales"], state["block_table"], state["case"]["n"],
                                       state["importance"], state["lse"])
    if state["workspace"] is None:
        state["workspace"] = torch.empty(spf.spf_score_paged_fp8_workspace_bytes([prompt]), dtype=torch.uint8, device="cuda")
    spf.spf_score_paged_fp8([prompt], state["workspace"], dev_status=state["status"])
    return dict(importance=state["importance"], lse=state["lse"])


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
    state["q_out"].copy_(_rotate(state["q"], state["rope"], pos).to(torch.bfloat16))
    k, v = _rotate(state["k"], state["rope"], pos), state["v"].float()
    for x, pool, scale in ((k, state["k_pool"], state["k_scale"]), (v, state["v_pool"], state["v_scale"])):
        block = pool.shape[2]
        at, off = state["block_table"][seq, pos // block].long(), pos % block
        if scale is None:
            pool[at, :, off] = x.to(torch.bfloat16)
            continue
        # scales: of the new tokens, and of the ones that a block had before the step
        heads, parts = scale.shape[1:]
        part = off // SCALE_TOKENS
        amax = torch.zeros((scale.shape[0], parts, heads), device="cuda")
        place = (at * parts + part)[:, None].expand(-1, heads)
        amax.view(-1, heads).scatter_reduce_(0, place, x.abs().amax(-1), "amax")
        before = state["seq_lens"].long() - state["row_start"].diff()
        here = state["block_table"].gather(1, (before // block).clamp(max=state["block_table"].shape[1] - 1)[:, None].long())[:, 0].long()
        there = (before % block) // SCALE_TOKENS
        partly = (before % SCALE_TOKENS) > 0
        here, there, left = here[partly], there[partly], (before % SCALE_TOKENS)[partly]
        was = scale[here, :, there]
        now = torch.maximum(was, _pow2_scale(amax[here, there]))
        cells = pool.view(pool.shape[0], heads, parts, SCALE_TOKENS, -1)
        held = cells[here, :, there].view(torch.float8_e4m3fn).float() * (was / now)[..., None, None]
        kept = torch.arange(SCALE_TOKENS, device="cuda")[None, None, :, None] < left[:, None, None, None]
        cells[here, :, there] = torch.where(kept, held.to(torch.float8_e4m3fn).view(torch.uint8), cells[here, :, there])
        fresh = _pow2_scale(amax[at, part])
        fresh[:] = torch.where((pos - pos % SCALE_TOKENS < before[seq])[:, None], torch.maximum(scale[at, :, part], fresh), fresh)
        scale[at, :, part] = fresh
        pool[at, :, off] = (x / fresh[..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return _appended(state)


def _gathered(pool, scale, table, length):
    """fp32 [sequences, heads, length, d] of a paged cache; what a table's unused entries point to is masked later."""
    x = pool[table.clamp(min=0).long()]                                # [seqs, blocks, heads, tokens, d]
    x = x.float() if scale is None else x.view(torch.float8_e4m3fn).float()
    if scale is not None:
        s = scale[table.clamp(min=0).long()]
        x = (x.view(*s.shape, SCALE_TOKENS, x.shape[-1]) * s[..., None, None]).view(x.shape)
    return x.transpose(1, 2).flatten(2, 3)[:, :, :length]


def _plain_attend(state):
    case = state["case"]
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    B, new = case["seqs"], state["max_new"]
    k = _gathered(state["k_pool"], state["k_scale"], state["block_table"], state["max_len"])
    v = _gathered(state["v_pool"], state["v_scale"], state["block_table"], state["max_len"])
    i = torch.arange(new, device="cuda")
    start, count = state["row_start"][:-1].long(), state["row_start"].diff()
    row = (start[:, None] + i).clamp(max=state["rows"] - 1)            # [seqs, new]; rows behind a sequence's are dropped below
    q = state["q"][row].float().view(B, new, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, d)
    last = state["seq_lens"].long()[:, None] - count[:, None] + i      # the position of a row, the last key that it sees
    z = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d)).view(B, Hkv, Hq // Hkv, new, -1)
    z.masked_fill_(torch.arange(k.shape[2], device="cuda") > last[:, None, None, :, None], float("-inf"))
    top = z.amax(-1, keepdim=True)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    # a sequence's own length hides what a shorter one has behind it; its values there are finite, so a zero weight is enough
    o = (p.flatten(2, 3) @ v).view(*p.shape[:-1], d) / total
    lse = (top + total.log())[..., 0]
    live = (i < count[:, None])
    state["out"][row[live]] = o.permute(0, 3, 1, 2, 4).reshape(B, new, Hq, d)[live].to(torch.bfloat16)
    state["lse"][row[live]] = lse.permute(0, 3, 1, 2).reshape(B, new, Hq)[live]
    return dict(out=state["out"], lse=state["lse"])


def _plain_score(state):
    case = state["case"]
    L, Hq, Hkv, d, m, n = (case[x] for x in ("L", "Hq", "Hkv", "d", "m", "n"))
    table = state["block_table"].long()
    s = state["scale"][:, table]
    k = state["pool"][:, table].view(torch.float8_e4m3fn).float()      # [L, blocks, heads, tokens, d]
    k = (k.view(*s.shape, SCALE_TOKENS, d) * s[..., None, None]).view(k.shape).transpose(1, 2).flatten(2, 3)[:, :, :n]
    z = (state["q"].float().view(L, Hkv, -1, d) @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    top = z.amax(-1, keepdim=True)
    z = z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    state["lse"].copy_((top + total.log()).view(L, Hq, m))
    state["importance"].copy_(z.div_(total).view(L * Hq, m, n).amax(0).mean(0))
    return dict(importance=state["importance"], lse=state["lse"])


# ---------------------------------------------------------------------------------------------- 64 bits
def _wide(pool, scale):
    if scale is None:
        return pool.double()
    x = pool.view(torch.float8_e4m3fn).to(torch.float32).double()
    return x * scale.double().repeat_interleave(SCALE_TOKENS, -1)[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "score":
        return _exact_score(case, s)
    old, new = _lengths(case)
    if case["op"] == "attend":
        return _exact_attend(case, s, old, new)
    return _exact_append(case, s, old, new)


def _exact_attend(case, s, old, new):
    d, group, block = case["d"], case["Hq"] // case["Hkv"], case["block"]
    out, lse = torch.zeros_like(s["out"], dtype=torch.float64), torch.zeros_like(s["lse"], dtype=torch.float64)
    row = 0
    for b, (before, count) in enumerate(zip(old, new)):
        ids = s["block_table"][b, :-(-(before + count) // block)].long()
        hidden = torch.arange(before + count, device="cuda")[None, :] > (before + torch.arange(count, device="cuda"))[:, None]
        for h in range(case["Hkv"]):
            k, v = (_wide(s[x + "_pool"][ids, h], None if s[x + "_scale"] is None else s[x + "_scale"][ids, h]).reshape(-1, d)[:before + count]
                    for x in "kv")
            for g in range(h * group, (h + 1) * group):
                z = s["q"][row:row + count, g].double() @ k.T / math.sqrt(d)
                z[hidden] = -math.inf
                lse[row:row + count, g] = torch.logsumexp(z, -1)
                out[row:row + count, g] = torch.exp(z - lse[row:row + count, g, None]) @ v
        row += count
    return dict(out=out, lse=lse)


def _exact_score(case, s):
    L, Hq, Hkv, d, m, n = (case[x] for x in ("L", "Hq", "Hkv", "d", "m", "n"))
    lse = torch.zeros((L, Hq, m), dtype=torch.float64, device="cuda")
    best = torch.zeros((m, n), dtype=torch.float64, device="cuda")
    ids = s["block_table"].long()
    for l in range(L):
        for h in range(Hkv):
            k = _wide(s["k_pools"][l][ids, h], s["k_scales"][l][ids, h]).reshape(-1, d)[:n]
            for g in range(h * Hq // Hkv, (h + 1) * Hq // Hkv):
                z = s["q"][l, g].double() @ k.T / math.sqrt(d)
                lse[l, g] = torch.logsumexp(z, -1)
                best = torch.maximum(best, torch.exp(z - lse[l, g, :, None]))
    return dict(importance=best.mean(0), lse=lse)


def _exact_append(case, s, old, new):
    """The values before they are rounded to the cache's type (8 bits: in units of the block's scale)."""
    d, block, half = case["d"], case["block"], case["d"] // 2
    bits8 = case["bits"] == 8
    powers = torch.tensor([2.0 ** e for e in range(-100, 128)], dtype=torch.float64, device="cuda")
    got = dict(q=torch.zeros_like(s["q_out"], dtype=torch.float64))
    for x in "kv":
        pool = s[x + "_pool"]
        got[x] = pool.view(torch.float8_e4m3fn).to(torch.float32).double() if bits8 else pool.double()
        if bits8:
            got[x + "_scale"] = s[x + "_scale"].double().clone()
    row = 0
    for b, (before, count) in enumerate(zip(old, new)):
        pos = torch.arange(before, before + count, device="cuda")
        cos, sin = s["rope"][pos, :half].double()[:, None], s["rope"][pos, half:].double()[:, None]
        turned = {}
        for x in "qk":
            a = s[x][row:row + count].double()
            turned[x] = torch.cat([a[..., :half] * cos - a[..., half:] * sin, a[..., half:] * cos + a[..., :half] * sin], -1)
        got["q"][row:row + count] = turned["q"]
        for x, y in (("k", turned["k"]), ("v", s["v"][row:row + count].double())):
            for first in range(before - before % SCALE_TOKENS, before + count, SCALE_TOKENS):
                lo, hi = max(first, before), min(first + SCALE_TOKENS, before + count)
                at, off = int(s["block_table"][b, first // block]), first % block
                part = y[lo - before:hi - before].transpose(0, 1)      # [heads, tokens, d]
                if not bits8:
                    got[x][at, :, lo % block:lo % block + hi - lo] = part
                    continue
                to = powers[torch.searchsorted(powers * E4M3_MAX, part.abs().amax((1, 2)))]
                if lo > first:
                    was = got[x + "_scale"][at, :, off // SCALE_TOKENS]
                    to = torch.maximum(to, was)
                    got[x][at, :, off:off + lo - first] *= (was / to)[:, None, None]
                got[x + "_scale"][at, :, off // SCALE_TOKENS] = to
                got[x][at, :, lo % block:lo % block + hi - lo] = part / to[:, None, None]
        row += count
    return got


# ---------------------------------------------------------------------------------------------- floors
def work(case):
    """Each input read once, each output written once: of the cache, the rows that the call is about."""
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    size = case["bits"] // 8
    if case["op"] == "score":
        L, m, n = case["L"], case["m"], case["n"]
        return {"bytes": L * Hkv * n * (d + 4 / SCALE_TOKENS) + L * Hq * m * (2 * d + 4) + 4 * n, "flops": 2.0 * L * Hq * m * n * d}
    old, new = _lengths(case)
    rows = sum(new)
    if case["op"] == "append":
        return {"bytes": rows * d * (4 * Hq + 2 * Hkv * (2 + size)) + 4 * d * max(a + b for a, b in zip(old, new)), "flops": 3.0 * rows * d * (Hq + Hkv)}
    keys = sum(a + b for a, b in zip(old, new))
    pairs = sum(b * a + b * (b + 1) // 2 for a, b in zip(old, new))
    return {"bytes": 2 * Hkv * keys * (d * size + (4 / SCALE_TOKENS if size == 1 else 0)) + rows * Hq * (4 * d + 4), "flops": 4.0 * Hq * d * pairs}
