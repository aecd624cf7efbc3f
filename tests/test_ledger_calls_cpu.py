"""Host-side checks of the calls on 4-bit caches and on the ledger beside a cache: what is refused, before anything could be launched (no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def spf():
    from paper_2603_02631_b200.build import build_library
    build_library()
    import paper_2603_02631_b200 as mod
    return mod


P = 1 << 20      # an aligned address that is never read


def _changed(struct, **fields):
    new = type(struct).from_buffer_copy(struct)
    for name, value in fields.items():
        setattr(new, name, value)
    return new


def _structs():
    from paper_2603_02631_b200 import binding as b
    return b, b._KvCache(P, P, P, P, 10, 256, 2, 64, 4), b._KvStep(2, 5, 1, 3, P, P, P)


BAD_CACHE = [(dict(k_pool=None), -1), (dict(v_pool=P + 8), -1), (dict(k_scale=None), -1), (dict(k_scale=None, v_scale=None), -1), (dict(k_scale=P + 8), -1),
             (dict(bits=5), -1), (dict(bits=-4), -1), (dict(bits=16), -1), (dict(n_pool_blocks=0), -1), (dict(block_tokens=64), -1),
             (dict(n_kv_heads=0), -1), (dict(head_dim=96), -2), (dict(n_pool_blocks=1 << 40), -2)]


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_caches_of_4_bits_are_checked_by_every_call(spf):
    b, cache, step = _structs()
    rows, ledger, options = b._Rows(P, 256, 64), b._KvLedger(P, P), b._AttendOptions(P, 4, 1, None, 0)
    cut = b._KvCut(2, 3, 2, 0, 0, P, P, P, P, P, None)
    calls = {
        "spf_kv_append": lambda c: spf.lib.spf_kv_append(ref(c), ref(step), None, ref(rows), ref(rows), None, None, 0, None, None),
        "spf_attend": lambda c: spf.lib.spf_attend(ref(c), ref(step), ref(rows), ref(b._Rows(2 * P, 256, 64)), 4, 0.0, None, P, 1 << 40, None, None),
        "spf_kv_weigh": lambda c: spf.lib.spf_kv_weigh(ref(c), ref(step), ref(rows), 4, 0.0, ref(options), ref(ledger), None, None, None),
        "spf_kv_evict": lambda c: spf.lib.spf_kv_evict(ref(c), ref(ledger), ref(cut), P, 1 << 40, None, None)}
    for who, call in calls.items():
        for fields, status in BAD_CACHE:
            assert call(_changed(cache, **fields)) == status, (who, fields)
            assert spf.spf_last_error().startswith(who)
        assert call(None) == -1
    assert spf.lib.spf_kv_append(ref(_changed(cache, bits=0, k_scale=P, v_scale=P)), ref(_changed(step, n_rows=0)), None, None, None, None, None, 0, None, None) == 0


def test_weigh_refuses(spf):
    b, cache, step = _structs()
    q, ledger, attend = b._Rows(P, 256, 64), b._KvLedger(P, P), b._AttendOptions(P, 4, 1, None, 0)
    options = b._KvWeighOptions(1.0, 0, None)

    def call(cache=cache, step=step, q=q, heads=4, attend=attend, ledger=ledger, options=options):
        return spf.lib.spf_kv_weigh(ref(cache), ref(step), ref(q), heads, 0.0, ref(attend), ref(ledger), ref(options), None, None)

    for fields in (dict(n_seqs=0), dict(n_rows=-1), dict(max_new=0), dict(table_stride=0), dict(row_start=None), dict(seq_lens=None), dict(block_table=None)):
        assert call(step=_changed(step, **fields)) == -1, fields
        assert spf.spf_last_error().startswith("spf_kv_weigh")
    for fields in (dict(data=None), dict(data=P + 2), dict(stride_row=4), dict(stride_head=-8)):
        assert call(q=_changed(q, **fields)) == -1, fields
    for fields in (dict(lse=None), dict(lse_stride_row=0), dict(lse_stride_head=0), dict(lse_stride_row=-1)):
        assert call(attend=_changed(attend, **fields)) == -1, fields
    for fields in (dict(decay=-0.5), dict(decay=float("nan")), dict(decay=float("inf")), dict(last_rows=-1)):
        assert call(options=_changed(options, **fields)) == -1, fields
    for fields in (dict(weight=None), dict(weight=P + 2), dict(position=P + 1)):
        assert call(ledger=_changed(ledger, **fields)) == -1, fields
    assert call(step=None) == -1 and call(q=None) == -1 and call(attend=None) == -1 and call(ledger=None) == -1
    assert call(heads=0) == -1 and call(heads=5) == -2
    assert call(step=_changed(step, n_rows=0)) == 0


def test_evict_refuses(spf):
    b, cache, _ = _structs()
    ledger, cut = b._KvLedger(P, None), b._KvCut(2, 3, 2, 0, 0, P, P, P, P, P, None)

    def call(cut=cut, ledger=ledger, ws=P, ws_bytes=1 << 40):
        return spf.lib.spf_kv_evict(ref(cache), ref(ledger), ref(cut), ws, ws_bytes, None, None)

    for fields in (dict(n_seqs=0), dict(n_seqs=(1 << 20) + 1), dict(table_stride=0), dict(to_stride=0), dict(n_first=-1), dict(n_recent=-1), dict(seq_lens=None),
                   dict(block_table=None), dict(keep=None), dict(to_table=None), dict(to_lens=None)):
        assert call(_changed(cut, **fields)) == -1, fields
        assert spf.spf_last_error().startswith("spf_kv_evict")
    for fields in (dict(n_seqs=1 << 20), dict(table_stride=1 << 23), dict(to_stride=1 << 23)):
        assert call(_changed(cut, **fields)) == -2, fields
    assert call(cut=None) == -1 and call(ledger=None) == -1 and call(ledger=_changed(ledger, weight=None)) == -1
    need = spf.lib.spf_kv_evict_workspace_bytes(ref(cache), 2, 2)
    assert need >= 2 * 2 * (2 * 256 + 1) * 4
    assert call(ws=None) == -3 and call(ws=P + 16) == -3 and call(ws_bytes=need - 1) == -3
    assert spf.lib.spf_kv_evict_workspace_bytes(ref(cache), 0, 2) == 0 and spf.lib.spf_kv_evict_workspace_bytes(ref(cache), 2, 0) == 0


def test_tensors_are_checked(spf):
    import torch
    pool, scale = torch.zeros(2, 2, 128, 32, dtype=torch.uint8), torch.zeros(2, 2, 128, 2, dtype=torch.bfloat16)
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    cache, step, ledger = spf.KvCache(pool, pool, scale, scale), spf.KvStep(i, i[:1], i[None]), spf.KvLedger(torch.zeros(2, 2, 128))
    with pytest.raises(TypeError):                                            # host tensors
        spf.spf_kv_append(cache, step, x, x)
    with pytest.raises(TypeError):
        spf.spf_kv_weigh(cache, step, x, torch.zeros(4, 2), ledger)
    with pytest.raises(TypeError):
        spf.spf_kv_evict(cache, ledger, i, i[None], i, i[None], i, pool)
    with pytest.raises(ValueError):
        spf.spf_kv_append(spf.KvCache(pool, pool, scale), step, x, x)         # one of the two scales
