"""Refusals and size queries of the operators beside the decoding step (no kernel is launched, so no GPU is needed)."""
import ctypes
import os
import subprocess

import pytest

from conftest import ROOT

NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED, ALIGN = 1, 2, 3, 6, 7, 9
vp = lambda a: ctypes.c_void_p(a) if a else None  # noqa: E731


@pytest.fixture(scope="module")
def rdk():
    from paper_2506_03206_amd import rdk as mod
    if not os.path.exists(mod.LIB_PATH):
        from paper_2506_03206_amd import build
        build.build()
    return mod


def test_topk_refusals(rdk):
    L, need = rdk.lib(), ctypes.c_size_t()

    def call(B=4, N=1000, k=16, t=1.0, kind=1, x=0x1000, ld=1000, ids=0x2000, values=0x3000, lse=0x4000, ws=0x5000, bytes=1 << 40):
        d = rdk.TopkDesc(B=B, N=N, k=k, temperature=t)
        return L.rdk_topk(ctypes.byref(d), vp(x), kind, ld, vp(ids), vp(values), vp(lse), vp(ws), bytes, None)

    d = rdk.TopkDesc(B=1024, N=151936, k=64, temperature=1.0)
    assert L.rdk_topk_workspace_bytes(ctypes.byref(d), 2, ctypes.byref(need)) == 0 and need.value >= 256
    assert L.rdk_topk_workspace_bytes(ctypes.byref(d), 2, None) == NULL
    assert L.rdk_topk_workspace_bytes(None, 2, ctypes.byref(need)) == NULL
    assert L.rdk_topk(None, vp(0x1000), 1, 10, vp(0x2000), vp(0x3000), None, vp(0x5000), 1 << 30, None) == NULL
    for kw in ({"B": 0}, {"B": -1}, {"N": 0}, {"k": 0}, {"k": 17, "N": 16, "ld": 16}, {"t": 0.0}, {"t": -1.0}, {"t": float("inf")},
               {"t": float("nan")}, {"ld": 999}):
        assert call(**kw) == SHAPE, kw
    assert call(kind=3) == DTYPE and call(kind=-1) == DTYPE
    assert call(k=129) == UNSUPPORTED and call(kind=0, t=2.0) == UNSUPPORTED
    for name in ("x", "ids", "values", "ws"):
        assert call(**{name: 0}) == NULL, name
    assert call(x=0x1008) == ALIGN and call(ws=0x5004) == ALIGN
    assert call(bytes=0) == WORKSPACE


def test_distill_refusals(rdk):
    L, need = rdk.lib(), ctypes.c_size_t()
    names = ("z", "ids", "top", "loss", "stats", "dz", "ws")

    def call(which, B=4, n=1000, K=16, t=1.0, kind=1, ldz=1000, ldd=1000, lse=0, weight=0, bytes=1 << 40, **at):
        p = {name: 0x100000 * (i + 1) for i, name in enumerate(names)}
        p.update(at)
        d = rdk.DistillDesc(B=B, n=n, K=K, temperature=t)
        head = (ctypes.byref(d), None, vp(p["z"]), kind, ldz, vp(p["ids"]), vp(p["top"]))
        if which == "loss":
            return L.rdk_distill_loss(*head, vp(lse), vp(weight), vp(p["loss"]), vp(p["stats"]), vp(p["ws"]), bytes, None)
        if which == "grad":
            return L.rdk_distill_grad(*head, vp(p["stats"]), vp(weight), vp(p["dz"]), ldd, None)
        return L.rdk_distill_loss_grad(*head, vp(lse), vp(weight), vp(p["loss"]), vp(p["stats"]), vp(p["dz"]), ldd, vp(p["ws"]), bytes, None)

    d = rdk.DistillDesc(B=2048, n=32064, K=64, temperature=1.0)
    assert L.rdk_distill_workspace_bytes(ctypes.byref(d), 2, ctypes.byref(need)) == 0 and need.value >= 256
    assert L.rdk_distill_workspace_bytes(ctypes.byref(d), 0, ctypes.byref(need)) == UNSUPPORTED
    assert L.rdk_distill_workspace_bytes(None, 1, ctypes.byref(need)) == NULL
    for which in ("loss", "grad", "both"):
        for kw in ({"B": 0}, {"n": 0}, {"K": 0}, {"t": 0.0}, {"t": float("inf")}, {"ldz": 999}):
            assert call(which, **kw) == SHAPE, (which, kw)
        assert call(which, kind=5) == DTYPE and call(which, kind=0) == UNSUPPORTED and call(which, K=129) == UNSUPPORTED
        for name in ("z", "ids", "top"):
            assert call(which, **{name: 0}) == NULL, (which, name)
        assert call(which, z=0x100004) == ALIGN
        if which != "grad":
            assert call(which, loss=0) == NULL and call(which, ws=0) == NULL and call(which, ws=0x700008) == ALIGN
            assert call(which, bytes=16) == WORKSPACE
        if which != "both":
            assert call(which, stats=0) == NULL
        assert call(which, stats=0x500004) == ALIGN
        if which != "loss":
            assert call(which, dz=0) == NULL and call(which, ldd=999) == SHAPE and call(which, dz=0x600002) == ALIGN
            assert call(which, dz=0x100000, ldd=1008) == SHAPE                       # z itself, but other strides
            assert call(which, dz=0x100010) == SHAPE                                 # overlaps z


def test_beam_select_refusals(rdk):
    L, need = rdk.lib(), ctypes.c_size_t()

    def call(G=2, W=4, N=1000, K=4, eos=7, kind=1, ld=1000, x=0x100000, scores=0x200000, finished=0x300000, so=0x400000, parent=0x500000,
             token=0x600000, fo=0x700000, ws=0x800000, bytes=1 << 40):
        d = rdk.BeamDesc(G=G, W=W, N=N, K=K, eos=eos)
        return L.rdk_beam_select(ctypes.byref(d), vp(x), kind, ld, vp(scores), vp(finished), vp(so), vp(parent), vp(token), vp(fo), vp(ws),
                                 bytes, None)

    d = rdk.BeamDesc(G=16, W=8, N=128256, K=8, eos=7)
    assert L.rdk_beam_select_workspace_bytes(ctypes.byref(d), 2, ctypes.byref(need)) == 0 and need.value >= 256
    assert L.rdk_beam_select_workspace_bytes(ctypes.byref(d), 9, ctypes.byref(need)) == DTYPE
    assert L.rdk_beam_select_workspace_bytes(ctypes.byref(d), 1, None) == NULL
    for kw in ({"G": 0}, {"W": 0}, {"N": 0}, {"K": 0}, {"eos": -2}, {"eos": 1000}, {"ld": 999}, {"eos": -1}, {"so": 0x200008},
               {"fo": 0x300004}):
        assert call(**kw) == SHAPE, kw
    assert call(W=65) == UNSUPPORTED and call(K=129) == UNSUPPORTED and call(W=64, N=1 << 25, ld=1 << 25) == UNSUPPORTED
    for name in ("x", "scores", "so", "parent", "token", "ws"):
        assert call(**{name: 0}) == NULL, name
    assert call(x=0x100008) == ALIGN and call(ws=0x800004) == ALIGN and call(bytes=0) == WORKSPACE


def test_reorder_refusals(rdk):
    L = rdk.lib()

    def state(src=0x10000000, dst=0x20000000, ss=4096, ds=4096, segments=1, bytes=4096, sp=0, dp=0):
        return rdk.State(src=src, dst=dst, src_stride=ss, dst_stride=ds, segments=segments, segment_bytes=bytes, src_pitch=sp, dst_pitch=dp)

    def call(s=None, G=2, W=4, K=4, parent=0x1000, count=1):
        return L.rdk_beam_reorder(G, W, K, vp(parent), ctypes.byref(s) if s is not None else None, count, None)

    assert call(state(), G=0) == SHAPE and call(state(), W=0) == SHAPE and call(state(), K=0) == SHAPE and call(state(), count=-1) == SHAPE
    assert call(state(), W=65) == UNSUPPORTED and call(state(), K=65) == UNSUPPORTED
    assert call(state(), parent=0) == NULL and call(None) == NULL and call(state(src=0)) == NULL and call(state(dst=0)) == NULL
    assert call(None, count=0) == 0                                                   # nothing to reorder
    assert call(state(segments=0)) == 0 and call(state(bytes=0, src=0, dst=0)) == 0     # a state of which nothing is filled
    for s in (state(bytes=-1), state(segments=-1), state(ss=4095), state(ds=100), state(ss=-4096), state(ss=1 << 60), state(ds=1 << 62),
              state(segments=2, bytes=2048, sp=2047, dp=2048), state(segments=2, bytes=2048, sp=2048, dp=2049),
              state(segments=1 << 40, bytes=16, sp=1 << 40, dp=16),
              state(dst=0x10000010),                                                  # overlaps its source
              state(dst=0x10000000, ds=8192),                                         # in place, but other strides
              state(dst=0x10000000, segments=2, bytes=1024, sp=2048, dp=1024)):
        assert call(s) == SHAPE
    assert call(state(dst=0x10000000), K=3) == SHAPE                                  # in place, but fewer rows


def test_limits_of_a_launch(rdk):
    """More rows than a launch has workgroups for, and temperatures whose reciprocal is no number."""
    L, need = rdk.lib(), ctypes.c_size_t()

    def topk(B, t=1.0):
        d = rdk.TopkDesc(B=B, N=10, k=3, temperature=t)
        return L.rdk_topk_workspace_bytes(ctypes.byref(d), 1, ctypes.byref(need))

    def distill(B, t=1.0):
        d = rdk.DistillDesc(B=B, n=10, K=3, temperature=t)
        return L.rdk_distill_workspace_bytes(ctypes.byref(d), 1, ctypes.byref(need))

    def beam(G, W):
        d = rdk.BeamDesc(G=G, W=W, N=10, K=3, eos=-1)
        return L.rdk_beam_select_workspace_bytes(ctypes.byref(d), 1, ctypes.byref(need))

    assert topk((1 << 24) - 1) == 0 and topk(1 << 24) == UNSUPPORTED
    assert distill((1 << 22) - 1) == 0 and distill(1 << 22) == UNSUPPORTED
    assert beam(((1 << 24) - 1) // 3, 3) == 0 and beam(1 << 18, 64) == UNSUPPORTED
    for call in (topk, distill):
        assert call(4, 1.2e-38) == 0 and call(4, 1e-39) == SHAPE and call(4, 3e38) == 0


def test_descriptors_match_the_header(rdk, tmp_path):
    src = tmp_path / "layout.c"
    mirrors = {"rdk_topk_desc_t": rdk.TopkDesc, "rdk_distill_desc_t": rdk.DistillDesc, "rdk_beam_desc_t": rdk.BeamDesc, "rdk_state_t": rdk.State}
    lines = ['  printf("%s %%zu\\n", sizeof(%s));' % (t, t) for t in mirrors]
    lines += ['  printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (t, f, t, f) for t, m in mirrors.items() for f, _ in m._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rdk.h"\nint main(void) {\n' + "\n".join(lines) + "\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        key, value = line.rsplit(" ", 1)
        t, _, f = key.partition(".")
        assert (getattr(mirrors[t], f).offset if f else ctypes.sizeof(mirrors[t])) == int(value), key
