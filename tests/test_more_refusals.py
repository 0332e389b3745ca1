"""What the entry points for norms with rotation, pages and logits refuse, on the host, before anything is launched (CPU: the addresses
are never used)."""
import ctypes as C

import pytest

import paper_2510_15312_amd as vf
from paper_2510_15312_amd.generate import _Adjust

L, P = vf.lib, C.c_void_p(4096)   # some address
ARG, UNSUPPORTED, CAP, OK = vf.VF_ERR_ARG, vf.VF_ERR_UNSUPPORTED, vf.VF_ERR_CAP, vf.VF_OK


def _addresses(n):
    return [C.c_void_p(4096 + 64 * i) for i in range(n)]


# ---- norms with rotation -------------------------------------------------------------------------

def _norm(ptrs=None, norm=None, **kw):
    base = dict(dtype=vf.VF_BF16, n_q_heads=4, n_kv_heads=2, head_dim=64, rotary_dim=64, pairs=vf.VF_ROTARY_HALF, total_rows=3,
                max_positions=10, pool_pages=2, pad=0, q_stride=512, k_stride=512, v_stride=512, q_out_stride=256)
    gains = dict(q_gain_dev=4096, k_gain_dev=4096, q_gain_stride=0, k_gain_stride=64, eps=1e-6, pad=0)
    base.update(kw), gains.update(norm or {})
    return L.vf_norm_rotary_append(C.byref(vf.vf_rotary_args(**base)), C.byref(vf.vf_head_norm(**gains)),
                                   *(ptrs or [P] * 6 + [C.c_void_p(8192), P]), None)


@pytest.mark.parametrize("norm,code", [
    (dict(eps=0.0), ARG), (dict(eps=-1e-6), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(q_gain_stride=-64), ARG),
    (dict(k_gain_stride=32), ARG), (dict(q_gain_stride=63), ARG), (dict(q_gain_stride=1 << 21), ARG), (dict(k_gain_stride=66), UNSUPPORTED),
    (dict(q_gain_dev=4100), UNSUPPORTED), (dict(k_gain_dev=4104), UNSUPPORTED)])
def test_norms(norm, code):
    assert _norm(norm=norm) == code and L.vf_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), ARG), (dict(n_q_heads=0), ARG), (dict(n_kv_heads=257), ARG), (dict(head_dim=96), UNSUPPORTED), (dict(rotary_dim=72), UNSUPPORTED),
    (dict(pairs=2), ARG), (dict(total_rows=-1), ARG), (dict(max_positions=0), ARG), (dict(pool_pages=0), ARG), (dict(q_stride=255), ARG),
    (dict(v_stride=132), UNSUPPORTED), (dict(ptrs=[P] * 8), ARG)])
def test_norms_with_what_the_rotation_refuses(kw, code):
    assert _norm(**kw) == code and b"vf_norm_rotary_append" in L.vf_last_error()


def test_norms_null_and_empty():
    for i in range(8):
        assert _norm(ptrs=[P] * i + [None] + [P] * (7 - i)) == ARG, i
    assert _norm(ptrs=[None] * 8, total_rows=0) == OK
    assert L.vf_norm_rotary_append(None, C.byref(vf.vf_head_norm(eps=1.0)), *[P] * 8, None) == ARG
    assert L.vf_norm_rotary_append(C.byref(vf.vf_rotary_args()), None, *[P] * 8, None) == ARG


# ---- pages -----------------------------------------------------------------------------------------

def _args(**kw):
    base = dict(n_seqs=3, max_pages=4, table_stride=4, pool_pages=9, free_entries=9, pad=0)
    base.update(kw)
    return vf.vf_pages_args(**base)


def _fork(ptrs=None, forks=2, **kw):
    return L.vf_pages_fork(C.byref(_args(**kw)), forks, *(ptrs or _addresses(12)), None)


def _keep(ptrs=None, **kw):
    return L.vf_pages_keep(C.byref(_args(**kw)), *(ptrs or _addresses(10)), None)


def _compact(ptrs=None, room=5, out_stride=4, **kw):
    return L.vf_pages_compact(C.byref(_args(**kw)), room, out_stride, *(ptrs or _addresses(10)), None)


@pytest.mark.parametrize("call", [_fork, _keep, _compact])
@pytest.mark.parametrize("kw,code", [
    (dict(n_seqs=0), ARG), (dict(n_seqs=vf.VF_PACKED_MAX_SEQS + 1), ARG), (dict(max_pages=0), ARG), (dict(table_stride=3), ARG),
    (dict(pool_pages=0), ARG), (dict(pool_pages=vf.VF_PAGES_MAX_POOL + 1), UNSUPPORTED), (dict(free_entries=-1), ARG), (dict(free_entries=1 << 30), ARG),
    (dict(n_seqs=4096, max_pages=(1 << 18) + 1, table_stride=1 << 20), UNSUPPORTED), (dict(max_pages=1 << 30, table_stride=1 << 30), ARG)])
def test_sizes_of_pages(call, kw, code):
    assert call(**kw) == code and L.vf_last_error()


@pytest.mark.parametrize("call,n", [(_fork, 12), (_keep, 10), (_compact, 10)])
def test_null_arrays(call, n):
    for i in range(n):
        p = _addresses(n)
        p[i] = None
        assert call(ptrs=p) == ARG, i


def test_forks():
    assert _fork(forks=-1) == ARG and _fork(forks=vf.VF_PACKED_MAX_SEQS + 1) == ARG
    p = _addresses(12)
    assert _fork(ptrs=p[:8] + [p[3]] + p[9:]) == ARG            # kv_len over len
    assert _fork(ptrs=p[:9] + [p[5]] + p[10:]) == ARG           # n_free in place
    assert L.vf_pages_fork(None, 1, *p, None) == ARG


def test_keeps():
    p = _addresses(10)
    assert _keep(ptrs=p[:6] + [p[0]] + p[7:]) == ARG and _keep(ptrs=p[:6] + [p[1]] + p[7:]) == ARG and _keep(ptrs=p[:7] + [p[3]] + p[8:]) == ARG
    assert L.vf_pages_keep(None, *p, None) == ARG


def test_compactions():
    p = _addresses(10)
    assert _compact(room=0) == ARG and _compact(out_stride=3) == ARG and _compact(room=vf.VF_PAGES_MAX_POOL + 1) == UNSUPPORTED
    assert _compact(ptrs=p[:4] + [p[2]] + p[5:]) == ARG and _compact(ptrs=p[:7] + [p[2]] + p[8:]) == ARG
    assert _compact(ptrs=p[:3] + [p[1]] + p[4:], out_stride=5) == ARG       # the table in place with another stride
    assert L.vf_pages_compact(None, 1, 4, *p, None) == ARG


def _copy(ptrs=None, **kw):
    base = dict(n_layers=2, page_bytes=4096, src_pages=3, dst_pages=5, max_copies=4, pad=0, src_layer_stride=3 * 4096, dst_layer_stride=5 * 4096)
    base.update(kw)
    return L.vf_pages_copy(C.byref(vf.vf_copy_args(**base)), *(ptrs or [P] * 4), None)


@pytest.mark.parametrize("kw,code", [
    (dict(n_layers=0), ARG), (dict(page_bytes=0), ARG), (dict(page_bytes=(1 << 30) + 16), ARG), (dict(src_pages=0), ARG), (dict(dst_pages=0), ARG),
    (dict(max_copies=-1), ARG), (dict(src_layer_stride=2 * 4096), ARG), (dict(dst_layer_stride=4 * 4096), ARG), (dict(page_bytes=4088), UNSUPPORTED),
    (dict(src_layer_stride=3 * 4096 + 8), UNSUPPORTED), (dict(ptrs=[C.c_void_p(4104), P, P, P]), UNSUPPORTED),
    (dict(n_layers=1 << 30, page_bytes=1 << 16, src_layer_stride=1 << 20, dst_layer_stride=1 << 20), UNSUPPORTED)])
def test_copies(kw, code):
    assert _copy(**kw) == code and L.vf_last_error()


def test_more_copies_than_indexes_reach():
    assert _copy(max_copies=(1 << 30) + 1) == ARG and _copy(ptrs=[P, P, None, P], max_copies=1 << 30) == ARG
    assert b"NULL" in L.vf_last_error()


def test_copies_null_and_empty():
    for i in range(4):
        assert _copy(ptrs=[P] * i + [None] + [P] * (3 - i)) == ARG, i
    assert _copy(ptrs=[None] * 4, max_copies=0) == OK
    assert L.vf_pages_copy(None, *[P] * 4, None) == ARG


# ---- logits ----------------------------------------------------------------------------------------

def _logits(ptrs=None, **kw):
    base = dict(dtype=vf.VF_F32, n_seqs=2, total_rows=3, vocab=100, max_history=5, bias_entries=4, mask_rows=3, pad=0, in_stride=100, out_stride=100,
                history_stride=5, mask_stride=4)
    base.update(kw)
    return L.vf_logits_adjust(C.byref(vf.vf_logits_args(**base)), *(ptrs or _addresses(13)), None)


def _without(*which, n=13):
    p = _addresses(n)
    for i in which:
        p[i] = None
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), ARG), (dict(n_seqs=0), ARG), (dict(n_seqs=vf.VF_PACKED_MAX_SEQS + 1), ARG), (dict(total_rows=-1), ARG),
    (dict(total_rows=vf.VF_PACKED_MAX_ROWS + 1), ARG), (dict(vocab=0), ARG), (dict(vocab=vf.VF_LOGITS_MAX_VOCAB + 1, in_stride=1 << 30, out_stride=1 << 30), ARG),
    (dict(in_stride=99), ARG), (dict(out_stride=99), ARG), (dict(max_history=-1), ARG), (dict(max_history=vf.VF_LOGITS_MAX_HISTORY + 1, history_stride=1 << 30), ARG),
    (dict(history_stride=4), ARG), (dict(bias_entries=-1), ARG), (dict(bias_entries=vf.VF_LOGITS_MAX_BIASES + 1), ARG), (dict(mask_rows=-1), ARG), (dict(mask_stride=3), ARG),
    (dict(ptrs=_without(0)), ARG), (dict(ptrs=_without(1)), ARG), (dict(ptrs=_without(2)), ARG),
    (dict(ptrs=_without(5)), ARG),                              # a history without lengths
    (dict(ptrs=_without(4)), ARG),                              # prompt lengths without a history
    (dict(ptrs=_without(9)), ARG), (dict(ptrs=_without(10)), ARG),
    (dict(ptrs=_without(12), mask_rows=2), ARG),                # fewer masks than rows
    (dict(ptrs=[P, C.c_void_p(8192), P] + _addresses(10), dtype=vf.VF_BF16), ARG),      # in place with another type
    (dict(ptrs=[P, C.c_void_p(8192), P] + _addresses(10), out_stride=104), ARG),        # or stride
    (dict(ptrs=[C.c_void_p(4098)] + _addresses(12)), UNSUPPORTED), (dict(ptrs=_addresses(2) + [C.c_void_p(8194)] + _addresses(10)), UNSUPPORTED)])
def test_logits(kw, code):
    assert _logits(**kw) == code and L.vf_last_error()


def test_logits_null_and_empty():
    assert L.vf_logits_adjust(None, *[P] * 13, None) == ARG
    assert _logits(ptrs=[None] * 13, total_rows=0) == OK


@pytest.mark.parametrize("penalties", [(0.0, 0.0, 0.0), (-1.0, 0.1, 0.1), (float("nan"), 0.0, 0.0), (1.0, 0.0), (1.0, 0.0, 0.0, 0.0)])
def test_penalties_of_generate(penalties):
    with pytest.raises(ValueError, match="repetition"):
        _Adjust(penalties, None, None, [1, 2], 10, 20, "cpu")
