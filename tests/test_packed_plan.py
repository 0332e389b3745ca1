"""Kernel and parts that vf_attention_packed chooses, held against kept timings of every kernel and many splits (host only)."""
import ctypes as C
import os

import paper_2510_15312_amd as vf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _calls():
    for line in open(os.path.join(ROOT, "profiles", "packed_attention_plan_timings.txt")):
        if line.startswith("#"):
            continue
        name, shape, sizes, times = (x.split() for x in line.split("|"))
        timed = {}
        for t in times:
            where, us = t.split(":")
            timed[tuple(int(x) for x in where.split("/"))] = float(us)
        yield name[0], shape[0], [int(x) for x in shape[1:]], [int(x) for x in sizes], timed


def _args(dtype, shape, sizes):
    (hq, hkv, hd), (n, rows, max_rows, max_keys) = shape, sizes
    return vf.vf_packed_args(vf.VF_F32 if dtype == "f32" else vf.VF_BF16, hq, hkv, hd, n, rows, max_rows, max_keys, 1 << 20, 1 << 12,
                             1 << 12, 0.0, hq * hd, hq * hd)


def _choice(args):
    kernel, parts = C.c_int(), C.c_int()
    assert vf.lib.vf_debug_packed_plan(C.byref(args), C.byref(kernel), C.byref(parts)) == vf.VF_OK
    return kernel.value, parts.value


def test_the_choice_costs_little():
    losses = {}
    for name, dtype, shape, sizes, timed in _calls():
        kernel, parts = _choice(_args(dtype, shape, sizes))
        near = min((k for k in timed if k[0] == kernel), key=lambda k: abs(k[1] - parts))
        losses[name] = timed[near] / min(timed.values()) - 1
    assert len(losses) > 150
    assert sum(losses.values()) / len(losses) < 0.025, losses
    assert max(losses.values()) < 0.25, sorted(losses.items(), key=lambda x: -x[1])[:5]


def test_every_kernel_is_chosen_somewhere_and_workspaces_stay_small():
    seen = set()
    for _, dtype, shape, sizes, _ in _calls():
        args = _args(dtype, shape, sizes)
        kernel, parts = _choice(args)
        seen.add((dtype, kernel, parts > 1))
        need = vf.lib.vf_attention_packed_workspace(C.byref(args))
        assert (need > 0) == (parts > 1) and need <= 16 * sizes[1] * shape[0] * (shape[2] + 4) * 4 + 4 * sizes[1]
    assert {("bf16", k, s) for k in (0, 1, 2) for s in (False, True)} | {("f32", 0, True), ("f32", 2, False), ("f32", 2, True)} <= seen


def test_single_tokens_take_the_kernel_of_sixteen_items():
    for rows in (1, 5, 400):
        for keys in (1, 64, 5000, 200000):
            assert _choice(_args("bf16", (16, 1, 128), (rows, rows, 1, keys)))[0] == 2


def test_the_largest_calls_have_a_kernel():
    """Tiles of 16 items would be more workgroups than a launch takes: 2^20 rows of 256 key heads."""
    for dtype in ("bf16", "f32"):
        for n, rows in ((1, 1 << 20), (4096, 1 << 20), (4096, 1 << 12)):
            args = _args(dtype, (256, 256, 64), (n, rows, rows, rows))
            kernel, parts = _choice(args)
            tiles = rows // (16 if kernel == 2 else 128) + n
            assert tiles * parts * 256 <= 0x7fffff
