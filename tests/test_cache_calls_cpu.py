"""Host-side checks of the calls on the draft model's cache: what is refused, before anything could be launched (no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def spf():
    from paper_2603_02631_b200.build import build_library
    build_library()
    import paper_2603_02631_b200 as mod
    return mod


P = 1 << 20      # an aligned address that is never read


def _structs():
    from paper_2603_02631_b200 import binding as b
    cache = b._KvCache(P, P, None, None, 10, 256, 2, 64)
    step = b._KvStep(2, 5, 1, 3, P, P, P)
    return b, cache, step


def _changed(struct, **fields):
    new = type(struct).from_buffer_copy(struct)
    for name, value in fields.items():
        setattr(new, name, value)
    return new


BAD_CACHE = [(dict(k_pool=None), -1), (dict(v_pool=P + 8), -1), (dict(k_scale=P), -1), (dict(k_scale=P + 2, v_scale=P), -1), (dict(n_pool_blocks=0), -1),
             (dict(block_tokens=64), -1), (dict(block_tokens=200), -1), (dict(n_kv_heads=0), -1), (dict(head_dim=96), -2),
             (dict(n_pool_blocks=1 << 40), -2), (dict(n_pool_blocks=(1 << 31) // 512), -2)]
BAD_STEP = [dict(n_seqs=0), dict(n_rows=-1), dict(max_new=0), dict(table_stride=0), dict(row_start=None), dict(seq_lens=None), dict(block_table=None)]
BAD_ROWS = [dict(data=None), dict(data=P + 2), dict(stride_row=4), dict(stride_head=-8)]


def test_append_refuses(spf):
    b, cache, step = _structs()
    k, q = b._Rows(P, 128, 64), b._Rows(P, 256, 64)
    rope = b._Rope(P, None, 100, 64, 0)

    def call(cache=cache, step=step, rope=rope, k=k, v=k, q=q, q_out=q, heads=4):
        ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return spf.lib.spf_kv_append(ref(cache), ref(step), ref(rope), ref(k), ref(v), ref(q), ref(q_out), heads, None, None)

    for fields, status in BAD_CACHE:
        assert call(cache=_changed(cache, **fields)) == status, fields
        assert spf.spf_last_error().startswith("spf_kv_append")
    for fields in BAD_STEP:
        assert call(step=_changed(step, **fields)) == -1, fields
    for fields in BAD_ROWS:
        for name in ("k", "v", "q", "q_out"):
            assert call(**{name: _changed(q, **fields)}) == -1, (name, fields)
    assert call(cache=None) == -1 and call(step=None) == -1 and call(k=None) == -1 and call(v=None) == -1
    assert call(q=None) == -1 and call(q_out=None) == -1 and call(heads=0) == -1
    assert call(q_out=_changed(q, stride_row=32)) == -1                       # rows of the output overlap
    assert call(q_out=_changed(q, stride_head=32)) == -1
    assert call(q_out=_changed(q, stride_row=512)) == -1                      # in place, but with other strides
    for fields in (dict(table=None), dict(table=P + 4), dict(n_positions=0), dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=80)):
        assert call(rope=_changed(rope, **fields)) == -1, fields
    assert call(step=_changed(step, n_rows=0)) == 0                           # nothing to append: nothing is launched
    assert spf.spf_status_string(-7) not in ("", "ok", "unknown status")


def test_append_checks_its_tensors(spf):
    import torch
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    pool = torch.zeros(2, 2, 128, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        spf.spf_kv_append(spf.KvCache(pool, pool), spf.KvStep(i, i[:1], i[None]), x, x)   # host tensors
    with pytest.raises(ValueError):
        spf.spf_kv_append(spf.KvCache(pool, pool, i), spf.KvStep(i, i[:1], i[None]), x, x)  # one of the two scales


def test_attend_refuses(spf):
    b, cache, step = _structs()
    q, out = b._Rows(P, 256, 64), b._Rows(2 * P, 256, 64)
    options = b._AttendOptions(P, 4, 1, None, 0)

    def call(cache=cache, step=step, q=q, out=out, heads=4, options=options, ws=P, ws_bytes=1 << 40):
        ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return spf.lib.spf_attend(ref(cache), ref(step), ref(q), ref(out), heads, 0.0, ref(options), ws, ws_bytes, None, None)

    for fields, status in BAD_CACHE:
        assert call(cache=_changed(cache, **fields)) == status, fields
        assert spf.spf_last_error().startswith("spf_attend")
    for fields in BAD_STEP:
        assert call(step=_changed(step, **fields)) == -1, fields
    for fields in BAD_ROWS:
        for name in ("q", "out"):
            assert call(**{name: _changed(q, **fields)}) == -1, (name, fields)
    assert call(cache=None) == -1 and call(step=None) == -1 and call(q=None) == -1 and call(out=None) == -1
    assert call(heads=0) == -1 and call(heads=5) == -2
    assert call(out=q) == -1                                                  # in place
    assert call(out=_changed(out, stride_head=32)) == -1                      # heads of the output overlap
    for fields in (dict(lse_stride_row=0), dict(lse_stride_head=0), dict(lse_stride_row=-1)):
        assert call(options=_changed(options, **fields)) == -1, fields
    assert call(step=_changed(step, n_rows=0)) == 0                           # nothing to do: nothing is launched
    assert spf.lib.spf_attend_workspace_bytes(ctypes.byref(_changed(cache, head_dim=96)), 4, 1) == 0
    assert spf.lib.spf_attend_workspace_bytes(ctypes.byref(cache), 4, 0) == 0
    assert spf.lib.spf_attend_workspace_bytes(ctypes.byref(cache), 3, 1) == 0


def test_score_paged_fp8_refuses(spf):
    b, _, _ = _structs()
    ptrs = (ctypes.c_void_p * 2)(P, 2 * P)
    odd = (ctypes.c_void_p * 2)(P, P + 2)
    none = (ctypes.c_void_p * 2)(P, None)
    lp = lambda x: ctypes.cast(x, ctypes.POINTER(ctypes.c_void_p))  # noqa: E731
    shape = b._Shape(2, 4, 2, 64, 8, 0.0)
    good = b._PagedFp8Prompt(1000, lp(ptrs), lp(ptrs), 10, 256, P, P, P, None)

    def call(prompt, shape=shape):
        arr = (b._PagedFp8Prompt * 1)(prompt)
        return spf.lib.spf_score_paged_fp8(ctypes.byref(shape), arr, 1, P, 1 << 40, None, None)

    for fields in (dict(n_tokens=0), dict(k_pools=lp(none)), dict(k_scales=None), dict(k_scales=lp(none)), dict(k_scales=lp(odd)), dict(n_pool_blocks=0),
                   dict(block_tokens=64), dict(block_tokens=200), dict(block_table=None), dict(q=None), dict(importance=None)):
        assert call(_changed(good, **fields)) == -1, fields
    assert call(good, b._Shape(2, 4, 2, 96, 8, 0.0)) == -2
    arr = (b._PagedFp8Prompt * 1)(good)
    assert spf.lib.spf_score_paged_fp8(ctypes.byref(shape), arr, 1, None, 0, None, None) == -3
    assert spf.lib.spf_score_paged_fp8_workspace_bytes(ctypes.byref(shape), arr, 1) > 0
