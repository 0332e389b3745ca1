"""ctypes binding of libvf.so: argument marshalling only.

Functions carry the names of the C entry points (include/vf.h).  torch is used
for device memory and for the current HIP stream; every step of the path runs
in the library's kernels.  There is no fallback: if the library is missing the
import fails.
"""
import ctypes as C
import functools
import os

import torch  # first: brings the HIP runtime the library links against into the process

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvf.so")

VF_OK, VF_ERR_ARG, VF_ERR_CAP, VF_ERR_HIP, VF_ERR_UNSUPPORTED = 0, -1, -2, -3, -4
VF_F32, VF_BF16 = 0, 1
VF_GREEDY, VF_STOCHASTIC = 0, 1
VF_PENDING = -1
VF_MAX_BATCH, VF_MAX_DRAFTS = 32, 32
VF_TOPK_MAX = 8
VF_ACCEPT_STATIC_MAX_ROWS = 512
VF_OPT_FAST_PATH = 1
VF_OPT_PERSISTENT = 2
VF_PACKED_MAX_SEQS, VF_PACKED_MAX_ROWS = 4096, 1 << 20
VF_ROTARY_HALF, VF_ROTARY_INTERLEAVED = 0, 1
VF_PAGES_MAX_POOL = 1 << 18
VF_LOGITS_MAX_VOCAB, VF_LOGITS_MAX_HISTORY, VF_LOGITS_MAX_BIASES = 1 << 24, 1 << 24, 1 << 28
VF_ROTARY_UNSCALED, VF_ROTARY_POSITIONS, VF_ROTARY_BASE, VF_ROTARY_RAMP = 0, 1, 2, 3

EXPORTS = [
    "vf_last_error", "vf_model_packed_bytes", "vf_model_create", "vf_model_destroy",
    "vf_seq_state_bytes", "vf_kv_bytes", "vf_seq_create", "vf_seq_destroy", "vf_seq_set_len",
    "vf_seq_set_pending", "vf_seq_get_state", "vf_seq_note_len", "vf_kv_read", "vf_kv_write", "vf_prefill_chunk", "vf_verify",
    "vf_accept", "vf_accept_static", "vf_profile", "vf_profile_read", "vf_set_option", "vf_stream_read",
    "vf_reuse_select", "vf_reuse_pool_init", "vf_reuse_pool_update", "vf_reuse_pool_extend",
    "vf_verify_tree", "vf_accept_tree", "vf_prefill_chunk_topk", "vf_draft_suffix_match",
    "vf_pages_assign", "vf_rotary_table", "vf_rotary_append", "vf_attention_packed_workspace", "vf_attention_packed",
    "vf_norm_rotary_append", "vf_pages_fork", "vf_pages_keep", "vf_pages_compact", "vf_pages_copy", "vf_logits_adjust",
]
SITES = ["qkv", "o", "gateup", "down", "head", "attn", "small", "accept", "step"]


class VfError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"vf error {code}: {msg}")
        self.code = code


class vf_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_q_heads", "n_kv_heads", "head_dim",
                                         "d_ffn", "vocab", "dtype")] + \
               [("rope_theta", C.c_float), ("rms_eps", C.c_float)] + \
               [(n, C.c_int32) for n in ("tie_embeddings", "qkv_bias", "max_rows", "max_positions")]


class vf_layer_w(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "wq", "wk", "wv", "bq", "bk", "bv", "wo",
                                          "ffn_norm", "w_gate", "w_up", "w_down")]


class vf_weights(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("lm_head", C.c_void_p), ("final_norm", C.c_void_p),
                ("layers", C.POINTER(vf_layer_w))]


class vf_accept_params(C.Structure):
    _fields_ = [("mode", C.c_int32), ("temperature", C.c_float), ("q_dev", C.c_void_p),
                ("u_dev", C.c_void_p)]


class vf_reuse_pool(C.Structure):
    _fields_ = [("tokens", C.c_int32 * VF_MAX_DRAFTS)] + \
               [(n, C.c_int32) for n in ("len", "age", "max_age", "cap")]


class vf_rotary_plan(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rotary_dim", "max_positions", "scaling", "pad")] + \
               [(n, C.c_double) for n in ("theta", "factor", "low", "high", "trained", "magnitude")]


class vf_rotary_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_q_heads", "n_kv_heads", "head_dim", "rotary_dim", "pairs",
                                         "total_rows", "max_positions", "pool_pages", "pad")] + \
               [(n, C.c_int64) for n in ("q_stride", "k_stride", "v_stride", "q_out_stride")]


class vf_head_norm(C.Structure):
    _fields_ = [("q_gain_dev", C.c_void_p), ("k_gain_dev", C.c_void_p), ("q_gain_stride", C.c_int32), ("k_gain_stride", C.c_int32),
                ("eps", C.c_float), ("pad", C.c_int32)]


class vf_pages_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_seqs", "max_pages", "table_stride", "pool_pages", "free_entries", "pad")]


class vf_copy_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "page_bytes", "src_pages", "dst_pages", "max_copies", "pad")] + \
               [(n, C.c_int64) for n in ("src_layer_stride", "dst_layer_stride")]


class vf_logits_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_seqs", "total_rows", "vocab", "max_history", "bias_entries", "mask_rows", "pad")] + \
               [(n, C.c_int64) for n in ("in_stride", "out_stride", "history_stride", "mask_stride")]


class vf_packed_args(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("dtype", "n_q_heads", "n_kv_heads", "head_dim", "n_seqs", "total_rows",
                                         "max_rows", "max_keys", "pool_pages", "max_pages", "table_stride")] + \
               [("scale", C.c_float)] + [(n, C.c_int64) for n in ("q_stride", "out_stride")]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it first (python -m paper_2510_15312_amd.build)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, sz = C.c_void_p, C.c_int32, C.c_size_t
    sig = {
        "vf_last_error": (C.c_char_p, []),
        "vf_model_packed_bytes": (sz, [C.POINTER(vf_config)]),
        "vf_model_create": (C.c_int, [C.POINTER(vf_config), C.POINTER(vf_weights), vp, sz, vp, C.POINTER(vp)]),
        "vf_model_destroy": (C.c_int, [vp]),
        "vf_seq_state_bytes": (sz, [vp]),
        "vf_kv_bytes": (sz, [vp, C.c_int, C.c_int]),
        "vf_seq_create": (C.c_int, [vp, vp, sz, C.c_int, C.c_int, C.c_int, vp, vp, vp, C.POINTER(vp)]),
        "vf_seq_destroy": (C.c_int, [vp]),
        "vf_seq_set_len": (C.c_int, [vp, C.c_int, vp]),
        "vf_seq_set_pending": (C.c_int, [vp, i32, vp]),
        "vf_seq_get_state": (C.c_int, [vp, C.POINTER(i32), C.POINTER(i32), vp]),
        "vf_seq_note_len": (C.c_int, [vp, C.c_int]),
        "vf_kv_read": (C.c_int, [vp, vp, C.c_int, C.c_int, C.c_int, vp, vp, vp]),
        "vf_kv_write": (C.c_int, [vp, vp, C.c_int, C.c_int, C.c_int, vp, vp, vp]),
        "vf_prefill_chunk": (C.c_int, [vp, vp, vp, C.c_int, C.c_int, vp, C.c_int, vp, C.c_float, vp]),
        "vf_verify": (C.c_int, [vp, C.POINTER(vp), C.c_int, vp, C.POINTER(i32), vp, vp]),
        "vf_accept": (C.c_int, [vp, C.POINTER(vp), C.c_int, vp, C.POINTER(i32), C.POINTER(vf_accept_params),
                                vp, vp, vp, vp, vp]),
        "vf_accept_static": (C.c_int, [vp, C.POINTER(vp), C.c_int, vp, C.POINTER(i32), C.POINTER(vf_accept_params),
                                       vp, vp, vp, vp, vp]),
        "vf_set_option": (C.c_int, [vp, C.c_int, C.c_int]),
        "vf_profile": (C.c_int, [vp, C.c_int]),
        "vf_stream_read": (C.c_int, [vp, C.POINTER(sz), vp]),
        "vf_profile_read": (C.c_int, [vp, C.POINTER(C.c_float), C.POINTER(i32)]),
        "vf_draft_suffix_match": (C.c_int, [C.POINTER(i32), C.c_int, C.c_int, C.c_int, C.c_int, C.POINTER(i32)]),
        "vf_prefill_chunk_topk": (C.c_int, [vp, vp, vp, C.c_int, C.c_int, vp, vp, C.c_int, vp, C.c_float, vp]),
        "vf_verify_tree": (C.c_int, [vp, C.POINTER(vp), C.c_int, vp, C.POINTER(i32), C.POINTER(i32), vp, vp]),
        "vf_accept_tree": (C.c_int, [vp, C.POINTER(vp), C.c_int, vp, C.POINTER(i32), C.POINTER(i32),
                                     C.POINTER(vf_accept_params), vp, vp, vp, vp, vp, vp]),
        "vf_reuse_select": (C.c_int, [C.c_int, vp, C.POINTER(i32), vp, vp, vp, vp]),
        "vf_reuse_pool_init": (C.c_int, [C.POINTER(vf_reuse_pool), C.c_int, C.c_int]),
        "vf_reuse_pool_update": (C.c_int, [C.POINTER(vf_reuse_pool), C.POINTER(i32), C.c_int, C.c_int, C.c_int]),
        "vf_reuse_pool_extend": (C.c_int, [C.POINTER(vf_reuse_pool), C.POINTER(i32), C.c_int]),
        "vf_pages_assign": (C.c_int, [C.c_int] * 5 + [vp] * 11),
        "vf_rotary_table": (C.c_int, [C.POINTER(vf_rotary_plan), vp, vp]),
        "vf_rotary_append": (C.c_int, [C.POINTER(vf_rotary_args)] + [vp] * 9),
        "vf_attention_packed_workspace": (sz, [C.POINTER(vf_packed_args)]),
        "vf_attention_packed": (C.c_int, [C.POINTER(vf_packed_args)] + [vp] * 7 + [sz, vp]),
        "vf_norm_rotary_append": (C.c_int, [C.POINTER(vf_rotary_args), C.POINTER(vf_head_norm)] + [vp] * 9),
        "vf_pages_fork": (C.c_int, [C.POINTER(vf_pages_args), C.c_int] + [vp] * 13),
        "vf_pages_keep": (C.c_int, [C.POINTER(vf_pages_args)] + [vp] * 11),
        "vf_pages_compact": (C.c_int, [C.POINTER(vf_pages_args), C.c_int, C.c_int] + [vp] * 11),
        "vf_pages_copy": (C.c_int, [C.POINTER(vf_copy_args)] + [vp] * 5),
        "vf_logits_adjust": (C.c_int, [C.POINTER(vf_logits_args)] + [vp] * 14),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


lib = _load()


def _check(rc):
    if rc != VF_OK:
        raise VfError(rc, lib.vf_last_error().decode())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _stream_of(t):
    """The current stream of the tensor's device as an address.  A step's packed calls take a few microseconds each: through
    the stream object this alone is 2.8 of them, like this 0.1."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


class Model:
    """Handle of a packed model; keeps the device buffer it lives in alive."""

    def __init__(self, handle, cfg, buf):
        self.handle, self.cfg, self.buf = handle, cfg, buf

    def __del__(self):
        if getattr(self, "handle", None):
            lib.vf_model_destroy(self.handle)
            self.handle = None


class Seq:
    """Handle of a sequence; keeps its KV memory, block table and state alive."""

    def __init__(self, handle, model, kv, state, block_table, capacity):
        self.handle, self.model, self.kv, self.state = handle, model, kv, state
        self.block_table, self.capacity = block_table, capacity

    def __del__(self):
        if getattr(self, "handle", None):
            lib.vf_seq_destroy(self.handle)
            self.handle = None


def make_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab, dtype, rope_theta,
                rms_eps, max_rows, max_positions, qkv_bias=False, tie_embeddings=True):
    return vf_config(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, vocab,
                     VF_BF16 if dtype in ("bf16", VF_BF16) else VF_F32, rope_theta, rms_eps,
                     int(tie_embeddings), int(qkv_bias), max_rows, max_positions)


def vf_model_packed_bytes(cfg):
    n = lib.vf_model_packed_bytes(C.byref(cfg))
    if n == 0:
        raise VfError(VF_ERR_ARG, lib.vf_last_error().decode())
    return n


def vf_model_create(cfg, weights, device="cuda:0"):
    """weights: dict like workloads.make_weights but of torch DEVICE tensors (matrices in the
    model dtype, vectors float32)."""
    layers = (vf_layer_w * cfg.n_layers)()
    for l, lw in enumerate(weights["layers"]):
        for name, _ in vf_layer_w._fields_:
            setattr(layers[l], name, lw[name].data_ptr() if lw.get(name) is not None else None)
    lm = weights.get("lm_head")
    w = vf_weights(weights["embed"].data_ptr(), lm.data_ptr() if lm is not None else None,
                   weights["final_norm"].data_ptr(), layers)
    nbytes = vf_model_packed_bytes(cfg)
    buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    out = C.c_void_p()
    _check(lib.vf_model_create(C.byref(cfg), C.byref(w), _ptr(buf), nbytes, _stream(), C.byref(out)))
    return Model(out, cfg, buf)


def vf_kv_bytes(model, page_tokens, n):
    b = lib.vf_kv_bytes(model.handle, page_tokens, n)
    if b == 0:
        raise VfError(VF_ERR_ARG, lib.vf_last_error().decode())
    return b


def vf_seq_create(model, capacity, pool=None, block_table=None, device="cuda:0"):
    """Contiguous cache (pool None: allocated here) or paged (pool = uint8 tensor of
    vf_kv_bytes(model, 64, n_pages), block_table = int32 device tensor)."""
    state = torch.empty(lib.vf_seq_state_bytes(model.handle), dtype=torch.uint8, device=device)
    out = C.c_void_p()
    if pool is None:
        kv = torch.empty(vf_kv_bytes(model, 0, capacity), dtype=torch.uint8, device=device)
        rc = lib.vf_seq_create(model.handle, _ptr(kv), kv.numel(), 0, 0, capacity, None, _ptr(state),
                               _stream(), C.byref(out))
    else:
        kv = pool
        es = 2 if model.cfg.dtype == VF_BF16 else 4
        page_bytes = model.cfg.n_layers * 2 * model.cfg.n_kv_heads * 64 * model.cfg.head_dim * es
        rc = lib.vf_seq_create(model.handle, _ptr(kv), kv.numel(), 64, kv.numel() // page_bytes, capacity,
                               _ptr(block_table), _ptr(state), _stream(), C.byref(out))
    _check(rc)
    return Seq(out, model, kv, state, block_table, capacity)


def vf_seq_set_len(seq, n):
    _check(lib.vf_seq_set_len(seq.handle, n, _stream()))


def vf_seq_set_pending(seq, token):
    _check(lib.vf_seq_set_pending(seq.handle, token, _stream()))


def vf_seq_get_state(seq):
    a, b = C.c_int32(), C.c_int32()
    _check(lib.vf_seq_get_state(seq.handle, C.byref(a), C.byref(b), _stream()))
    return a.value, b.value


def vf_seq_note_len(seq, n):
    """Host only: tightens the host-side bound of the length to the true length n."""
    _check(lib.vf_seq_note_len(seq.handle, int(n)))


def vf_kv_read(model, seq, layer, t0, n):
    shape = (n, model.cfg.n_kv_heads, model.cfg.head_dim)
    k = torch.empty(shape, dtype=torch.float32, device=seq.state.device)
    v = torch.empty(shape, dtype=torch.float32, device=seq.state.device)
    _check(lib.vf_kv_read(model.handle, seq.handle, layer, t0, n, _ptr(k), _ptr(v), _stream()))
    return k, v


def vf_kv_write(model, seq, layer, t0, k, v):
    """k, v: float32 device tensors [n, n_kv_heads, head_dim]."""
    _check(lib.vf_kv_write(model.handle, seq.handle, layer, t0, k.shape[0], _ptr(k), _ptr(v), _stream()))


def vf_prefill_chunk(model, seq, tokens, logits_mode=0, logits_out=None, sample_first=False, u=None,
                     temperature=0.0):
    """tokens: int32 device tensor [n]."""
    _check(lib.vf_prefill_chunk(model.handle, seq.handle, _ptr(tokens), tokens.numel(), logits_mode,
                                _ptr(logits_out), int(sample_first), _ptr(u), temperature, _stream()))


def _batch(seqs, row_off):
    hs = (C.c_void_p * len(seqs))(*[s.handle for s in seqs])
    ro = (C.c_int32 * len(row_off))(*[int(r) for r in row_off])
    return hs, ro


def vf_verify(model, seqs, tokens, row_off, logits_out=None):
    """tokens: int32 device tensor [total_rows]; row_off: host ints [n_seqs + 1]."""
    hs, ro = _batch(seqs, row_off)
    _check(lib.vf_verify(model.handle, hs, len(seqs), _ptr(tokens), ro, _ptr(logits_out), _stream()))


def vf_accept(model, seqs, tokens, row_off, params, n_accept, out_tokens, y, logits=None):
    """params: list of (mode, temperature, q tensor or None, u tensor or None) per sequence;
    n_accept int32[n_seqs], out_tokens int32[total_rows], y int32[total_rows]: device tensors."""
    hs, ro = _batch(seqs, row_off)
    ps = (vf_accept_params * len(seqs))()
    for i, (mode, temp, q, u) in enumerate(params):
        ps[i] = vf_accept_params(mode, temp, q.data_ptr() if q is not None else None,
                                 u.data_ptr() if u is not None else None)
    _check(lib.vf_accept(model.handle, hs, len(seqs), _ptr(tokens), ro, ps, _ptr(logits), _ptr(n_accept),
                         _ptr(out_tokens), _ptr(y), _stream()))


def vf_accept_static(model, seqs, tokens, row_off, params, n_accept, out_tokens, y, logits=None):
    """vf_accept with the library's static device scratch; arguments as vf_accept."""
    hs, ro = _batch(seqs, row_off)
    ps = (vf_accept_params * len(seqs))()
    for i, (mode, temp, q, u) in enumerate(params):
        ps[i] = vf_accept_params(mode, temp, q.data_ptr() if q is not None else None,
                                 u.data_ptr() if u is not None else None)
    _check(lib.vf_accept_static(model.handle, hs, len(seqs), _ptr(tokens), ro, ps, _ptr(logits), _ptr(n_accept),
                                _ptr(out_tokens), _ptr(y), _stream()))


def vf_prefill_chunk_topk(model, seq, tokens, top_k, topk_logit, topk_id, sample_first=False, u=None,
                          temperature=0.0):
    """tokens int32[n] (device); topk_logit float32[n, top_k], topk_id int32[n, top_k]: device tensors."""
    _check(lib.vf_prefill_chunk_topk(model.handle, seq.handle, _ptr(tokens), tokens.numel(), int(top_k),
                                     _ptr(topk_logit), _ptr(topk_id), int(bool(sample_first)), _ptr(u),
                                     float(temperature), _stream()))


def vf_verify_tree(model, seqs, tokens, row_off, parents, logits_out=None):
    """As vf_verify; parents: host ints [total_rows], -1 for each sequence's first row, else the
    parent's row within the sequence."""
    hs, ro = _batch(seqs, row_off)
    par = (C.c_int32 * len(parents))(*[int(p) for p in parents])
    _check(lib.vf_verify_tree(model.handle, hs, len(seqs), _ptr(tokens), ro, par, _ptr(logits_out), _stream()))


def vf_accept_tree(model, seqs, tokens, row_off, parents, params, n_accept, out_tokens, y, path, logits=None):
    """As vf_accept, plus path int32[total_rows] (device): the rows of the accepted path."""
    hs, ro = _batch(seqs, row_off)
    par = (C.c_int32 * len(parents))(*[int(p) for p in parents])
    ps = (vf_accept_params * len(seqs))()
    for i, (mode, temp, q, u) in enumerate(params):
        ps[i] = vf_accept_params(mode, temp, q.data_ptr() if q is not None else None,
                                 u.data_ptr() if u is not None else None)
    _check(lib.vf_accept_tree(model.handle, hs, len(seqs), _ptr(tokens), ro, par, ps, _ptr(logits), _ptr(n_accept),
                              _ptr(out_tokens), _ptr(y), _ptr(path), _stream()))


def vf_draft_suffix_match(history, k, max_suffix, min_suffix=1):
    """history: host ints; returns the list of drafts (possibly empty)."""
    n = len(history)
    arr = (C.c_int32 * max(1, n))(*[int(t) for t in history])
    out = (C.c_int32 * VF_MAX_DRAFTS)()
    got = lib.vf_draft_suffix_match(arr, n, int(max_suffix), int(min_suffix), int(k), out)
    if got < 0:
        _check(got)
    return list(out[:got])


def vf_reuse_select(tokens, row_off, y, n_accept, seg):
    """tokens, y int32[total_rows], n_accept int32[n_seqs], seg int32[2 * n_seqs]: device tensors."""
    ro = (C.c_int32 * len(row_off))(*[int(r) for r in row_off])
    _check(lib.vf_reuse_select(len(row_off) - 1, _ptr(tokens), ro, _ptr(y), _ptr(n_accept), _ptr(seg), _stream()))


def vf_reuse_pool_init(max_age, cap=VF_MAX_DRAFTS):
    pool = vf_reuse_pool()
    _check(lib.vf_reuse_pool_init(C.byref(pool), int(max_age), int(cap)))
    return pool


def vf_reuse_pool_update(pool, drafts, seg_start, seg_len):
    """drafts: host ints, the drafts of the step the segment was found in."""
    arr = (C.c_int32 * max(1, len(drafts)))(*[int(t) for t in drafts])
    _check(lib.vf_reuse_pool_update(C.byref(pool), arr, len(drafts), int(seg_start), int(seg_len)))


def vf_reuse_pool_extend(pool, fresh):
    """Returns the drafts of the next step: the fresh ones, then the held segment if it fits."""
    arr = (C.c_int32 * VF_MAX_DRAFTS)(*[int(t) for t in fresh])
    n = lib.vf_reuse_pool_extend(C.byref(pool), arr, len(fresh))
    if n < 0:
        _check(n)
    return list(arr[:n])


def vf_profile(model, enable):
    _check(lib.vf_profile(model.handle, int(enable)))


def vf_profile_read(model):
    """{site: (total ms, launch groups)} since the last read."""
    ms = (C.c_float * len(SITES))()
    cnt = (C.c_int32 * len(SITES))()
    _check(lib.vf_profile_read(model.handle, ms, cnt))
    return {s: (ms[i], cnt[i]) for i, s in enumerate(SITES)}


def vf_stream_read(model):
    """Launches the read-every-weight yardstick kernel; returns the bytes it reads."""
    n = C.c_size_t(0)
    _check(lib.vf_stream_read(model.handle, C.byref(n), _stream()))
    return n.value


def vf_set_option(model, option, value):
    _check(lib.vf_set_option(model.handle, option, int(value)))


# ---- packed batches ----------------------------------------------------------------------------

def _refuse(what):
    raise VfError(VF_ERR_ARG, what)


_I32 = torch.int32


@functools.cache
def _device_count():
    return torch.cuda.device_count()


def _several_devices():
    return _device_count() > 1


def _device(name, t):
    """The number of a tensor's device, on which all others of the call have to be; None where there is one device only, so that
    `is_cuda` says the same (asking every tensor of a call for its number takes 0.5 us of the call's 8)."""
    if not t.is_cuda:
        _refuse(f"{name}: device tensor")
    return t.get_device() if _several_devices() else None


def _current_device():
    """The current device's number; None where there is no other."""
    return torch.cuda.current_device() if _device_count() > 1 else None


def _launch(dev, call, *args):
    """A call whose tensors are on device dev: where that is not the current one, it is for the call, as the default streams of all
    devices have one address."""
    if dev is None or _current_device() in (dev, None):
        return _check(call(*args))
    with torch.cuda.device(dev):
        _check(call(*args))


def _on(device):
    return " on the device" if device is None else f" on device {device}"


def _ints(name, t, n, device):
    """The address of an int32 device tensor of at least n entries one behind the other."""
    if t.dtype is not _I32 or not t.is_cuda or t.numel() < n or not t.is_contiguous() or device is not None and t.get_device() != device:
        _refuse(f"{name}: contiguous int32 tensor of {n} entries{_on(device)}")
    return t.data_ptr()


def _below_31_bits(what, *sizes):
    """Refuses sizes that the library's 32-bit fields would cut."""
    if max(sizes) > 0x7fffffff:
        _refuse(f"{what}: a size of {max(sizes)}")


def _rows(name, t, dtype, rows, heads, hd, device):
    """The row stride of a device tensor [rows, heads, hd] whose rows are contiguous."""
    if t.dtype is not dtype or t.shape != (rows, heads, hd) or not t.is_cuda or device is not None and t.get_device() != device:
        _refuse(f"{name}: tensor [{rows}, {heads}, {hd}] of {dtype}{_on(device)}")
    row, head, one = t.stride()
    if one != 1 or (heads > 1 and head != hd):
        _refuse(f"{name}: rows that are contiguous")
    return row if rows > 1 else max(row, heads * hd)


def _pool(t, hd, dtype, device):
    """(pages, kv heads) of one layer's pages, [pages, 2, kv heads, 64 * hd]."""
    s = t.shape
    if len(s) != 4 or s[1] != 2 or s[3] != 64 * hd or t.dtype is not dtype or not t.is_contiguous() or not t.is_cuda or device is not None and t.get_device() != device:
        _refuse(f"pool: contiguous tensor [pages, 2, kv heads, {64 * hd}] of {dtype}{_on(device)}")
    return s[0], s[2]


def _table(t, device):
    """(sequences, entries a sequence, stride) of a block table."""
    if t.dim() != 2 or t.dtype is not _I32 or not t.is_cuda or device is not None and t.get_device() != device:
        _refuse(f"block table: int32 tensor [sequences, pages]{_on(device)}")
    (n, m), (row, one) = t.shape, t.stride()
    if one != 1 and m > 1:
        _refuse("block table: rows that are contiguous")
    return n, m, row if n > 1 else max(row, m)


_DTYPES = {torch.bfloat16: VF_BF16, torch.float32: VF_F32}


def _dtype(t):
    code = _DTYPES.get(t.dtype)
    return _refuse(f"dtype {t.dtype}") if code is None else code


def kv_layer(model, pool, layer):
    """One layer of a pool of vf_kv_bytes(model, 64, n) bytes as the packed operators take it: a view
    [n, 2, n_kv_heads, 64 * head_dim] in the model's type."""
    c = model.cfg
    t = pool.view(torch.bfloat16 if c.dtype == VF_BF16 else torch.float32)
    return t.view(c.n_layers, -1, 2, c.n_kv_heads, 64 * c.head_dim)[layer]


def vf_pages_assign(lens, new, free_pages, n_free, block_table, row_off, pos, slot, kv_len, n_free_out):
    """int32 device tensors: lens, new [n], free_pages [any], n_free [1], block_table [n, pages]; results row_off [n + 1],
    pos, slot [total rows], kv_len [n], n_free_out [1], and the fresh entries of block_table."""
    dev = _device("lens", lens)
    n, m, stride = _table(block_table, dev)
    rows = pos.numel()
    _launch(dev, lib.vf_pages_assign, n, m, stride, rows, free_pages.numel(), _ints("lens", lens, n, dev), _ints("new", new, n, dev),
            _ints("free_pages", free_pages, 0, dev), _ints("n_free", n_free, 1, dev), block_table.data_ptr(),
            _ints("row_off", row_off, n + 1, dev), _ints("pos", pos, rows, dev), _ints("slot", slot, rows, dev),
            _ints("kv_len", kv_len, n, dev), _ints("n_free_out", n_free_out, 1, dev), _stream_of(lens))


def vf_rotary_table(rotary_dim, theta, max_positions, scaling=VF_ROTARY_UNSCALED, factor=1.0, low=0.0, high=0.0, trained=0.0,
                    magnitude=1.0, device="cuda:0"):
    """float32 [max_positions, rotary_dim / 2, 2]: cos and sin of every position's angles."""
    plan = vf_rotary_plan(int(rotary_dim), int(max_positions), int(scaling), 0, theta, factor, low, high, trained, magnitude)
    table = torch.empty((max(int(max_positions), 0), max(int(rotary_dim), 0) // 2, 2), dtype=torch.float32, device=device)
    _launch(_device("table", table), lib.vf_rotary_table, C.byref(plan), _ptr(table), _stream_of(table))
    return table


def _rotary_args(q, k, v, table, q_out, pool, pairs, dev):
    rows, hq, hd = q.shape
    dt = q.dtype
    pages, hkv = _pool(pool, hd, dt, dev)
    positions, half, two = table.shape
    if two != 2 or table.dtype is not torch.float32 or not table.is_contiguous() or not table.is_cuda or dev is not None and table.get_device() != dev:
        _refuse(f"table: contiguous float32 tensor [positions, rotary_dim / 2, 2]{_on(dev)}")
    return vf_rotary_args(_dtype(q), hq, hkv, hd, 2 * half, pairs, rows, positions, pages, 0,
                          _rows("q", q, dt, rows, hq, hd, dev), _rows("k", k, dt, rows, hkv, hd, dev),
                          _rows("v", v, dt, rows, hkv, hd, dev), _rows("q_out", q_out, dt, rows, hq, hd, dev))


def vf_rotary_append(q, k, v, table, pos, slot, q_out, pool, pairs=VF_ROTARY_HALF):
    """q, q_out [rows, q heads, hd], k, v [rows, kv heads, hd] (views of wider rows allowed), table of vf_rotary_table, pos and
    slot int32 [rows], pool: one layer's pages (kv_layer)."""
    dev = _device("q", q)
    args = _rotary_args(q, k, v, table, q_out, pool, pairs, dev)
    _launch(dev, lib.vf_rotary_append, C.byref(args), q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(),
            _ints("pos", pos, args.total_rows, dev), _ints("slot", slot, args.total_rows, dev), q_out.data_ptr(),
            pool.data_ptr(), _stream_of(q))


def _gain(name, t, heads, hd, dev):
    """(address, stride between heads) of gains [hd] or [heads, hd]; None: no gains."""
    if t is None:
        return None, 0
    if t.dtype is not torch.float32 or not t.is_cuda or not t.is_contiguous() or dev is not None and t.get_device() != dev or \
            tuple(t.shape) not in ((hd,), (heads, hd)):
        _refuse(f"{name}: contiguous float32 tensor [{hd}] or [{heads}, {hd}]{_on(dev)}")
    return t.data_ptr(), hd if t.dim() == 2 else 0


def vf_norm_rotary_append(q, k, v, q_gain, k_gain, eps, table, pos, slot, q_out, pool, pairs=VF_ROTARY_HALF):
    """As vf_rotary_append, with every head of q and k normalised first: x * gain / sqrt(mean x^2 + eps).  q_gain, k_gain: float32
    [hd] or [heads, hd], or None."""
    dev = _device("q", q)
    args = _rotary_args(q, k, v, table, q_out, pool, pairs, dev)
    (qg, qs), (kg, ks) = _gain("q_gain", q_gain, args.n_q_heads, args.head_dim, dev), _gain("k_gain", k_gain, args.n_kv_heads, args.head_dim, dev)
    norm = vf_head_norm(qg, kg, qs, ks, eps, 0)
    _launch(dev, lib.vf_norm_rotary_append, C.byref(args), C.byref(norm), q.data_ptr(), k.data_ptr(), v.data_ptr(), table.data_ptr(),
            _ints("pos", pos, args.total_rows, dev), _ints("slot", slot, args.total_rows, dev),
            q_out.data_ptr(), pool.data_ptr(), _stream_of(q))


def _packed_args(q, pool, block_table, out, max_rows, max_keys, scale, dev):
    rows, hq, hd = q.shape
    pages, hkv = _pool(pool, hd, q.dtype, dev)
    n, m, stride = _table(block_table, dev)
    q_stride = _rows("q", q, q.dtype, rows, hq, hd, dev)
    return vf_packed_args(_dtype(q), hq, hkv, hd, n, rows, max_rows, max_keys, pages, m, stride, scale, q_stride,
                          q_stride if out is None else _rows("out", out, q.dtype, rows, hq, hd, dev))


def vf_attention_packed_workspace(q, pool, block_table, max_rows, max_keys):
    """A workspace for vf_attention_packed with these arguments: uint8 device tensor."""
    n = lib.vf_attention_packed_workspace(C.byref(_packed_args(q, pool, block_table, None, max_rows, max_keys, 0.0, _device("q", q))))
    if n == C.c_size_t(-1).value:
        raise VfError(VF_ERR_ARG, lib.vf_last_error().decode())
    return torch.empty(n, dtype=torch.uint8, device=q.device)


def vf_attention_packed(q, pool, block_table, row_off, kv_len, out, max_rows, max_keys, workspace, scale=0.0):
    """q, out [rows, q heads, hd]; pool: one layer's pages; block_table int32 [n, pages]; row_off int32 [n + 1] and kv_len
    int32 [n] on the device; max_rows, max_keys: the host's bounds of a sequence's rows and keys."""
    dev = _device("q", q)
    args = _packed_args(q, pool, block_table, out, max_rows, max_keys, scale, dev)
    if workspace.dtype is not torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous() or dev is not None and workspace.get_device() != dev:
        _refuse(f"workspace: contiguous uint8 tensor{_on(dev)}")
    _launch(dev, lib.vf_attention_packed, C.byref(args), q.data_ptr(), pool.data_ptr(), block_table.data_ptr(),
            _ints("row_off", row_off, args.n_seqs + 1, dev), _ints("kv_len", kv_len, args.n_seqs, dev),
            out.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream_of(q))


# ---- requests that branch, are cut back or move --------------------------------------------------

def _pages_args(block_table, shares, free_entries, dev):
    (n, m, stride), pages = _table(block_table, dev), shares.numel()
    _below_31_bits("pages", n, stride, pages, free_entries)
    return vf_pages_args(n, m, stride, pages, free_entries, 0)


def vf_pages_fork(src, dst, tokens, lens, free_pages, n_free, block_table, shares, kv_len, n_free_out, copies, n_copies):
    """int32 device tensors: src, dst, tokens [forks], lens [n], free_pages [any], n_free [1], block_table [n, pages], shares [pool
    pages]; results kv_len [n], n_free_out [1], copies [forks, 2], n_copies [1], and what changes in block_table and shares."""
    dev = _device("lens", lens)
    a, forks = _pages_args(block_table, shares, free_pages.numel(), dev), src.numel()
    _below_31_bits("src", forks)
    _launch(dev, lib.vf_pages_fork, C.byref(a), forks, _ints("src", src, forks, dev), _ints("dst", dst, forks, dev), _ints("tokens", tokens, forks, dev),
            _ints("lens", lens, a.n_seqs, dev), _ints("free_pages", free_pages, 0, dev), _ints("n_free", n_free, 1, dev),
            block_table.data_ptr(), _ints("shares", shares, 1, dev), _ints("kv_len", kv_len, a.n_seqs, dev),
            _ints("n_free_out", n_free_out, 1, dev), _ints("copies", copies, 2 * forks, dev), _ints("n_copies", n_copies, 1, dev),
            _stream_of(lens))


def vf_pages_keep(lens, keep, free_pages, n_free, block_table, shares, kv_len, n_free_out, copies, n_copies):
    """int32 device tensors: lens, keep [n], n_free [1], and free_pages [any], block_table [n, pages], shares [pool pages], which change
    in place; results kv_len [n], n_free_out [1], copies [n, 2], n_copies [1]."""
    dev = _device("lens", lens)
    a = _pages_args(block_table, shares, free_pages.numel(), dev)
    _launch(dev, lib.vf_pages_keep, C.byref(a), _ints("lens", lens, a.n_seqs, dev), _ints("keep", keep, a.n_seqs, dev), _ints("free_pages", free_pages, 0, dev),
            _ints("n_free", n_free, 1, dev), block_table.data_ptr(), _ints("shares", shares, 1, dev),
            _ints("kv_len", kv_len, a.n_seqs, dev), _ints("n_free_out", n_free_out, 1, dev),
            _ints("copies", copies, 2 * a.n_seqs, dev), _ints("n_copies", n_copies, 1, dev), _stream_of(lens))


def vf_pages_compact(lens, block_table, shares, table_out, shares_out, free_out, n_free_out, moved, copies, n_copies):
    """int32 device tensors: lens [n], block_table [n, pages], shares [pool pages]; results table_out [n, pages] (block_table itself
    allowed), shares_out and free_out [pages of the new pool], n_free_out [1], moved [pool pages], copies [pool pages, 2], n_copies [1]."""
    dev = _device("lens", lens)
    a, room = _pages_args(block_table, shares, 0, dev), shares_out.numel()
    n, m, stride = _table(table_out, dev)
    if (n, m) != (a.n_seqs, a.max_pages):
        _refuse(f"table_out: int32 tensor [{a.n_seqs}, {a.max_pages}]{_on(dev)}")
    _below_31_bits("table_out", stride, room)
    _launch(dev, lib.vf_pages_compact, C.byref(a), room, stride, _ints("lens", lens, a.n_seqs, dev), block_table.data_ptr(), _ints("shares", shares, 1, dev),
            table_out.data_ptr(), _ints("shares_out", shares_out, 1, dev), _ints("free_out", free_out, room, dev),
            _ints("n_free_out", n_free_out, 1, dev), _ints("moved", moved, a.pool_pages, dev),
            _ints("copies", copies, 2 * min(a.pool_pages, room), dev), _ints("n_copies", n_copies, 1, dev), _stream_of(lens))


def _layers(name, t, dev):
    """(layers, pages, bytes a page, bytes between layers) of pages [layers, pages, 2, kv heads, 64 * hd], or of one layer's without the first."""
    shape, stride, es = t.shape, t.stride(), t.element_size()
    if not 4 <= len(shape) <= 5 or not t.is_cuda or dev is not None and t.get_device() != dev:
        _refuse(f"{name}: tensor [layers, pages, 2, kv heads, 64 * head_dim]{_on(dev)}")
    pages, a, b, c = shape[-4:]
    if stride[-4:] != (a * b * c, b * c, c, 1) and any(n > 1 and step != want for n, step, want in zip(shape[-4:], stride[-4:], (a * b * c, b * c, c, 1))):
        _refuse(f"{name}: layers that are contiguous")
    layers = shape[0] if len(shape) == 5 else 1
    return layers, pages, a * b * c * es, (stride[0] if layers > 1 else pages * a * b * c) * es


def vf_pages_copy(pools, copies, n_copies, to):
    """pools, to: [layers, pages, 2, kv heads, 64 * hd] of all layers (or one layer without that dimension), of one type, which may be the same;
    copies int32 [any, 2], n_copies int32 [1] on the device."""
    dev = _device("pools", pools)
    layers, pages, size, stride = _layers("pools", pools, dev)
    to_layers, to_pages, to_size, to_stride = (layers, pages, size, stride) if to is pools else _layers("to", to, dev)
    if to_layers != layers or to_size != size or to.dtype is not pools.dtype:
        _refuse("pools of other layers, heads or types")
    _below_31_bits("pools", layers, size, pages, to_pages, copies.numel())
    a = vf_copy_args(layers, size, pages, to_pages, copies.numel() // 2, 0, stride, to_stride)
    _launch(dev, lib.vf_pages_copy, C.byref(a), pools.data_ptr(), to.data_ptr(), _ints("copies", copies, 0, dev), _ints("n_copies", n_copies, 1, dev),
            _stream_of(pools))


# ---- logits ----------------------------------------------------------------------------------------

def _matrix(name, t, dtype, rows, columns, dev):
    """The row stride of a device tensor [rows, columns] whose rows are contiguous; rows or columns None: any number."""
    s, steps = t.shape, t.stride()
    if len(s) != 2 or t.dtype is not dtype or not t.is_cuda or rows is not None and s[0] != rows or columns is not None and s[1] != columns or \
            steps[1] != 1 and s[1] > 1 or dev is not None and t.get_device() != dev:
        _refuse(f"{name}: tensor [{'any' if rows is None else rows}, {'any' if columns is None else columns}] of {dtype}, rows that are contiguous{_on(dev)}")
    return steps[0] if s[0] > 1 else max(steps[0], s[1])


def vf_logits_adjust(logits, row_off, out, penalties=None, history=None, history_len=None, prompt_len=None, tokens=None, biases=None,
                     mask=None, mask_row=None):
    """logits [rows, vocab] in bfloat16 or float32, out [rows, vocab] in float32 (logits itself allowed), row_off int32 [n + 1];
    penalties float32 [n, 3] (repetition, presence, frequency), history int32 [n, any], history_len and prompt_len int32 [n], tokens
    int32 [rows], biases: int32 offsets [n + 1], int32 ids and float32 values [any]; mask int32 [any, at least vocab / 32] (a bit an id),
    mask_row int32 [rows].  What is None is left out."""
    dev, shape, n = _device("logits", logits), logits.shape, row_off.numel() - 1
    if len(shape) != 2:
        _refuse(f"logits: tensor [rows, vocab]{_on(dev)}")
    rows, vocab = shape
    in_stride, out_stride = _matrix("logits", logits, logits.dtype, rows, vocab, dev), _matrix("out", out, torch.float32, rows, vocab, dev)

    penalty = text = bits = None
    text_most = text_stride = masks = mask_stride = entries = 0
    if penalties is not None:
        if _matrix("penalties", penalties, torch.float32, n, 3, dev) != 3 and n > 1:
            _refuse(f"penalties: contiguous float32 tensor [{n}, 3]{_on(dev)}")
        penalty = penalties.data_ptr()
    if history is not None:
        text_stride, text_most, text = _matrix("history", history, _I32, n, None, dev), history.shape[1], history.data_ptr()
    lengths = None if history_len is None else _ints("history_len", history_len, n, dev)
    prompts = None if prompt_len is None else _ints("prompt_len", prompt_len, n, dev)
    if history is not None and text_most == 0:      # texts without a token, which have no address
        text = lengths = prompts = None
    if mask is not None:
        mask_stride, bits, (masks, words) = _matrix("mask", mask, _I32, None, None, dev), mask.data_ptr(), mask.shape
        if 32 * words < vocab or mask_row is None and masks < rows:
            _refuse(f"mask: a bit for each of {vocab} ids, and a row for each row without mask_row")
    bias_off = bias_id = bias = None
    if biases is not None:
        bias_off, bias_id, bias = biases
        entries = bias_id.numel()
        if bias.dtype is not torch.float32 or not bias.is_cuda or not bias.is_contiguous() or bias.numel() != entries or \
                dev is not None and bias.get_device() != dev:
            _refuse(f"biases: contiguous float32 tensor of {entries} entries{_on(dev)}")
        bias_off, bias_id, bias = _ints("bias_off", bias_off, n + 1, dev), _ints("bias_id", bias_id, 0, dev), bias.data_ptr()
    _below_31_bits("logits", n, rows, vocab, text_most, entries, masks)
    a = vf_logits_args(_dtype(logits), n, rows, vocab, text_most, entries, masks, 0, in_stride, out_stride, text_stride, mask_stride)
    _launch(dev, lib.vf_logits_adjust, C.byref(a), logits.data_ptr(), _ints("row_off", row_off, 1, dev), out.data_ptr(), penalty, text,
            lengths, prompts, None if tokens is None else _ints("tokens", tokens, rows, dev), bias_off, bias_id, bias, bits,
            None if mask_row is None else _ints("mask_row", mask_row, rows, dev), _stream_of(logits))
