"""spf_attend on steps drawn at random: shapes, lengths, layouts, masks, hints, scales, and garbage wherever no row looks."""
import math
import random

import pytest
import torch

from attend_reference import decoded, gpu_step, reference

pytestmark = pytest.mark.gpu


def draw(rng, bits):
    hkv, group, seqs = rng.choice([1, 2, 3, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 33]), rng.choice([1, 1, 2, 5, 17, 60])
    most = {"one": 1, "few": rng.randint(2, 9), "many": rng.randint(10, 400)}[rng.choice(["one", "few", "many"])]
    longest = rng.choice([70, 300, 1500, 9000, 40000 if seqs < 3 else 3000])
    old, new = [rng.randint(0, longest) for _ in range(seqs)], [rng.randint(rng.choice([0, 1, 1]), most) for _ in range(seqs)]
    new[0] = max(new[0], 1)
    s = gpu_step(group * hkv, hkv, rng.choice([64, 128]), rng.choice([128, 256, 384, 1024]), old, new, bits, seed=rng.randrange(1 << 30),
                 rows=sum(new) + rng.choice([0, 0, 3]), q_scale=rng.choice([0.0, 0.5, 1.0, 2.0]))
    gen = torch.Generator(device="cuda").manual_seed(rng.randrange(1 << 30))
    if bits == 8:
        kind = rng.choice(["", "far", "zero", "odd"])
        if kind == "far":
            s.v_scale.copy_(2.0 ** torch.randint(-100, 101, s.v_scale.shape, generator=gen, device="cuda").double())
        elif kind == "zero":
            zero = torch.rand(s.v_scale.shape, generator=gen, device="cuda") < 0.5
            s.v_scale[zero] = 2.0 ** -100
            s.v_pool.view(*s.v_scale.shape, 64, s.d)[zero] = 0
        elif kind == "odd":
            s.v_scale.mul_(3.0)
            s.k_scale.mul_(0.37)
    if rng.random() < 0.4:                                  # logits that go up and down along the keys
        steep, period = rng.choice([5.0, 40.0, 150.0]), rng.choice([0.001, 0.01, 0.1])
        for b, n in enumerate(a + c for a, c in zip(old, new)):
            pos = torch.arange(n, device="cuda")
            ramp, blocks, place = 2 * torch.sin(pos.float() * period), s.table[b].long()[pos // s.block], pos % s.block
            if bits == 16:
                s.k_pool[blocks, :, place, 3] = ramp[:, None].to(torch.bfloat16)
            else:
                raw = (ramp[:, None] / s.k_scale[blocks, :, place // 64]).clamp(-448, 448).to(torch.float8_e4m3fn)
                s.k_pool[blocks, :, place, 3] = raw.view(torch.uint8)
        s.q[..., 3] = steep * s.d ** 0.5 / 2
    first = [rng.choice([0, rng.randint(-5, a + c + 3)]) for a, c in zip(old, new)] if rng.random() < 0.4 else None
    return s, first, rng.random() < 0.75, rng.choice([max(new), max(new), 1, 1000, rng.randint(1, 40)])


def outputs(rng, s):
    """An output with rows outside, heads outside, or as a slice, and lse likewise; and what must stay as it is."""
    kind = rng.choice(["rows", "heads", "slice"])
    shape = {"rows": (s.rows, s.Hq, s.d), "heads": (s.Hq, s.rows, s.d), "slice": (s.rows, s.Hq + 2, s.d + 8)}[kind]
    whole = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
    out = {"rows": whole, "heads": whole.transpose(0, 1), "slice": whole[:, 1:-1, :s.d]}[kind]
    lse = torch.full((s.Hq, s.rows), 7.0, device="cuda").T if rng.random() < 0.5 else torch.full((s.rows, s.Hq), 7.0, device="cuda")
    return out, lse, (lambda: [whole[:, 0], whole[:, -1], whole[:, :, s.d:]] if kind == "slice" else [])


def compare(s, out, lse, first, causal):
    """As attend_reference.check, with three roundings more, which ordinary inputs do not show.  8-bit queries are two terms, off by
    2^-21 of their row's largest element: logits by that times the sum of |k|.  fp16 weights below 2^-14 are off by 2^-25 where the
    largest, p s_v the largest of the row, is 2^7 or more: each key by 2^-32 of that times its byte, 448 at most.  Outputs below bf16's
    normal range are off by 2^-134."""
    group, operand = s.Hq // s.Hkv, 2.0 ** -8 if s.k_scale is None else 2.0 ** -11
    for b, new in enumerate(s.new):
        if new == 0:
            continue
        at, n, lo = torch.arange(new, device="cuda"), s.old[b] + new, 0 if first is None else max(first[b], 0)
        for h in sorted({0, s.Hkv - 1}):
            part = slice(h * group, (h + 1) * group)
            want, want_lse, weight, terms = reference(s, b, h, lo, causal, None, at)
            got, got_lse = out[int(s.row_start[b]) + at][:, part].double(), lse[int(s.row_start[b]) + at][:, part].double()
            empty, extra = want_lse == -math.inf, 0.0
            if s.k_scale is not None:
                k, q = decoded(s.k_pool, s.k_scale, s.table[b], h, n), s.q[int(s.row_start[b]) + at][:, part].double()
                terms = terms + 2.0 ** -5 * q.abs().amax(-1) * k[lo:].abs().sum(-1).amax() / math.sqrt(s.d) if lo < n else terms
                scale = s.v_scale[s.table[b][:-(-n // s.block)].long(), h].double().repeat_interleave(64, -1).flatten()[:n]
                z = torch.einsum("tgd,nd->tgn", q, k) / math.sqrt(s.d)
                key = torch.arange(n, device="cuda")
                hidden = (key < lo)[None].expand(new, -1)
                if causal:
                    hidden = hidden | (key[None] > (s.old[b] + at)[:, None])
                z.masked_fill_(hidden[:, None], -math.inf)
                extra = (n * 2.0 ** -32 * 448 * (torch.exp(z - torch.where(empty, 0.0, want_lse)[..., None]) * scale).amax(-1))[..., None]
            off = terms * 2.0 ** -16 + 2.0 ** -20
            assert torch.equal(got_lse == -math.inf, empty) and (got[empty] == 0).all()
            assert ((got_lse - want_lse).abs() <= off + 2.0 ** -22 * want_lse.abs())[~empty].all(), (b, h)
            bound = 2.0 ** -8 * want.abs() + (operand + 2 * off[..., None]) * weight * (1 + 2.0 ** -8) + extra + 2.0 ** -134
            assert ((got - want).abs() <= bound).all(), (b, h, float(((got - want).abs() - bound).max()))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("seed", range(60))
def test_steps_drawn_at_random(seed, bits):
    import paper_2603_02631_b200 as spf
    rng = random.Random(100 * seed + bits)
    s, first, causal, hint = draw(rng, bits)
    used = torch.zeros((s.k_pool.shape[0], s.block), dtype=torch.bool, device="cuda")
    for b, n in enumerate(a + c for a, c in zip(s.old, s.new)):
        pos = torch.arange(n if s.new[b] else 0, device="cuda")
        pos = pos[pos >= (0 if first is None else first[b])]
        used[s.table[b].long()[pos // s.block], pos % s.block] = True
    clean = s.k_pool.clone(), s.v_pool.clone()
    for pool in (s.k_pool, s.v_pool):
        pool.masked_fill_(~used[:, None, :, None], rng.choice([float("nan"), float("inf"), -float("inf")]) if bits == 16 else rng.choice([0x7F, 0xFF]))
    out, lse, others = outputs(rng, s)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    cache, step = s.cache(spf), s.step(spf, hint)
    ws = torch.full((spf.spf_attend_workspace_bytes(cache, step, s.q) + 64,), 255, dtype=torch.uint8, device="cuda")
    f = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    spf.spf_attend(cache, step, s.q, out, ws[:-64], lse, f, causal, 0.0, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0 and (ws[-64:] == 255).all()
    rows = sum(s.new)
    assert all((x == 7.0).all() for x in [out[rows:], lse[rows:], *others()])
    s.k_pool.copy_(clean[0]), s.v_pool.copy_(clean[1])
    compare(s, out, lse, first, causal)
