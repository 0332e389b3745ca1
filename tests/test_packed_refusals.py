"""What the packed-batch entry points refuse, on the host, before anything is launched (CPU: the addresses are never used)."""
import ctypes as C

import pytest

import paper_2510_15312_amd as vf

L, P = vf.lib, C.c_void_p(4096)   # some address


def _pages(n=2, pages=4, stride=4, rows=8, entries=9, ptrs=None):
    return L.vf_pages_assign(n, pages, stride, rows, entries, *(ptrs or [C.c_void_p(4096 + 64 * i) for i in range(10)]), None)


@pytest.mark.parametrize("kw", [dict(n=0), dict(n=vf.VF_PACKED_MAX_SEQS + 1), dict(pages=0), dict(stride=3), dict(rows=-1),
                                dict(rows=vf.VF_PACKED_MAX_ROWS + 1), dict(entries=-1), dict(entries=1 << 30)])
def test_pages_sizes(kw):
    assert _pages(**kw) == vf.VF_ERR_ARG and L.vf_last_error()


def test_pages_null_and_aliased_arguments():
    full = [C.c_void_p(4096 + 64 * i) for i in range(10)]
    for i in range(10):
        assert _pages(ptrs=full[:i] + [None] + full[i + 1:]) == vf.VF_ERR_ARG, i
    assert _pages(ptrs=full[:8] + [full[0], full[9]]) == vf.VF_ERR_ARG     # kv_len over len
    assert _pages(ptrs=full[:9] + [full[3]]) == vf.VF_ERR_ARG              # n_free in place


def _plan(**kw):
    base = dict(rotary_dim=64, max_positions=100, scaling=vf.VF_ROTARY_UNSCALED, pad=0, theta=1e4, factor=1.0, low=1.0, high=4.0,
                trained=512.0, magnitude=1.0)
    base.update(kw)
    return vf.vf_rotary_plan(**base)


@pytest.mark.parametrize("kw", [
    dict(rotary_dim=0), dict(rotary_dim=24), dict(rotary_dim=144), dict(max_positions=0), dict(theta=0.0), dict(theta=float("nan")),
    dict(theta=float("inf")), dict(magnitude=float("nan")), dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.0),
    dict(scaling=2, factor=float("inf")), dict(scaling=3, high=1.0), dict(scaling=3, trained=0.0), dict(scaling=3, factor=-2.0),
    dict(scaling=3, low=float("nan"))])
def test_rotary_table(kw):
    assert L.vf_rotary_table(C.byref(_plan(**kw)), P, None) == vf.VF_ERR_ARG and L.vf_last_error()


def test_rotary_table_null():
    assert L.vf_rotary_table(None, P, None) == vf.VF_ERR_ARG and L.vf_rotary_table(C.byref(_plan()), None, None) == vf.VF_ERR_ARG


def _rotary(ptrs=None, **kw):
    base = dict(dtype=vf.VF_BF16, n_q_heads=4, n_kv_heads=2, head_dim=64, rotary_dim=64, pairs=vf.VF_ROTARY_HALF, total_rows=3,
                max_positions=10, pool_pages=2, pad=0, q_stride=512, k_stride=512, v_stride=512, q_out_stride=256)
    base.update(kw)
    return L.vf_rotary_append(C.byref(vf.vf_rotary_args(**base)), *(ptrs or [P] * 6 + [C.c_void_p(8192), P]), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), vf.VF_ERR_ARG), (dict(n_q_heads=0), vf.VF_ERR_ARG), (dict(n_kv_heads=-1), vf.VF_ERR_ARG),
    (dict(head_dim=96), vf.VF_ERR_UNSUPPORTED), (dict(rotary_dim=72), vf.VF_ERR_UNSUPPORTED), (dict(rotary_dim=8), vf.VF_ERR_UNSUPPORTED),
    (dict(rotary_dim=128), vf.VF_ERR_UNSUPPORTED), (dict(pairs=2), vf.VF_ERR_ARG), (dict(total_rows=-1), vf.VF_ERR_ARG),
    (dict(total_rows=vf.VF_PACKED_MAX_ROWS + 1), vf.VF_ERR_ARG), (dict(max_positions=0), vf.VF_ERR_ARG), (dict(pool_pages=0), vf.VF_ERR_ARG),
    (dict(q_stride=255), vf.VF_ERR_ARG), (dict(k_stride=64), vf.VF_ERR_ARG), (dict(v_stride=132), vf.VF_ERR_UNSUPPORTED),
    (dict(ptrs=[P] * 8), vf.VF_ERR_ARG),                                             # q in place with another stride
    (dict(ptrs=[C.c_void_p(4104)] + [P] * 5 + [C.c_void_p(8192), P]), vf.VF_ERR_UNSUPPORTED)])
def test_rotary(kw, code):
    assert _rotary(**kw) == code and L.vf_last_error()


def test_rotary_null_and_empty():
    for i in range(8):
        assert _rotary(ptrs=[P] * i + [None] + [P] * (7 - i)) == vf.VF_ERR_ARG, i
    assert _rotary(ptrs=[None] * 8, total_rows=0) == vf.VF_OK             # nothing to do
    assert L.vf_rotary_append(None, *[P] * 8, None) == vf.VF_ERR_ARG


def _attn(**kw):
    base = dict(dtype=vf.VF_BF16, n_q_heads=4, n_kv_heads=2, head_dim=64, n_seqs=2, total_rows=3, max_rows=2, max_keys=100,
                pool_pages=4, max_pages=2, table_stride=2, scale=0.0, q_stride=256, out_stride=256)
    base.update(kw)
    return vf.vf_packed_args(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=-1), vf.VF_ERR_ARG), (dict(n_q_heads=5), vf.VF_ERR_ARG), (dict(n_kv_heads=0), vf.VF_ERR_ARG),
    (dict(n_q_heads=512), vf.VF_ERR_ARG), (dict(head_dim=80), vf.VF_ERR_UNSUPPORTED), (dict(n_seqs=0), vf.VF_ERR_ARG),
    (dict(n_seqs=vf.VF_PACKED_MAX_SEQS + 1), vf.VF_ERR_ARG), (dict(total_rows=-1), vf.VF_ERR_ARG), (dict(max_rows=-1), vf.VF_ERR_ARG),
    (dict(max_keys=-1), vf.VF_ERR_ARG), (dict(pool_pages=0), vf.VF_ERR_ARG), (dict(max_pages=0), vf.VF_ERR_ARG),
    (dict(table_stride=1), vf.VF_ERR_ARG), (dict(scale=float("nan")), vf.VF_ERR_ARG), (dict(scale=-1.0), vf.VF_ERR_ARG), (dict(q_stride=255), vf.VF_ERR_ARG),
    (dict(out_stride=260), vf.VF_ERR_UNSUPPORTED)])
def test_attention(kw, code):
    a = _attn(**kw)
    assert L.vf_attention_packed(C.byref(a), *[P] * 7, 1 << 30, None) == code and L.vf_last_error()
    assert L.vf_attention_packed_workspace(C.byref(a)) == C.c_size_t(-1).value


def test_attention_null_alignment_and_empty():
    a = _attn()
    for i in range(6):
        assert L.vf_attention_packed(C.byref(a), *[P] * i, None, *[P] * (6 - i), 1 << 30, None) == vf.VF_ERR_ARG, i
    assert L.vf_attention_packed(C.byref(a), C.c_void_p(4100), *[P] * 6, 1 << 30, None) == vf.VF_ERR_UNSUPPORTED
    assert L.vf_attention_packed(None, *[P] * 7, 0, None) == vf.VF_ERR_ARG
    assert L.vf_attention_packed(C.byref(_attn(total_rows=0)), *[None] * 7, 0, None) == vf.VF_OK

def test_workspace_too_small_is_refused():
    # one token over a long context: its keys are split and meet in the workspace
    a = _attn(n_seqs=1, total_rows=1, max_rows=1, max_keys=100_000, pool_pages=2000, max_pages=2000, table_stride=2000)
    need = L.vf_attention_packed_workspace(C.byref(a))
    assert 0 < need < 1 << 30
    assert L.vf_attention_packed(C.byref(a), *[P] * 7, need - 1, None) == vf.VF_ERR_CAP
    assert L.vf_attention_packed(C.byref(a), *[P] * 6, None, need, None) == vf.VF_ERR_ARG
