"""Refusals and size queries of the log probability and embedding calls (no kernel is launched, so no GPU is needed)."""
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


def logprobs_call(rdk, which, B=4, N=1000, C=2, k=0, t=1.0, kind=1, ldx=1000, ldd=1000, bytes=1 << 40, **at):
    L = rdk.lib()
    names = ("x", "tokens", "logprob", "rank", "entropy", "top_ids", "top", "stats", "dx", "ws", "gl", "ge")
    p = {name: 0x100000 * (i + 1) for i, name in enumerate(names)}
    p.update(at)
    q = {name: vp(a) for name, a in p.items()}
    d = rdk.LogprobsDesc(B=B, N=N, C=C, k=k, temperature=t)
    head = (ctypes.byref(d), None, q["x"], kind, ldx, q["tokens"])
    if which == "forward":
        return L.rdk_logprobs(*head, q["logprob"], q["rank"], q["entropy"], q["top_ids"], q["top"], q["stats"], q["ws"], bytes, None)
    if which == "grad":
        return L.rdk_logprobs_grad(*head, q["stats"], q["gl"], q["ge"], q["dx"], ldd, None)
    return L.rdk_logprobs_step(*head, q["gl"], q["ge"], q["logprob"], q["entropy"], q["stats"], q["dx"], ldd, q["ws"], bytes, None)


@pytest.mark.parametrize("which", ["forward", "grad", "step"])
def test_logprobs_refusals(rdk, which):
    call = lambda **kw: logprobs_call(rdk, which, **kw)  # noqa: E731
    for kw in ({"B": 0}, {"B": -3}, {"N": 0}, {"C": 0}, {"C": -1}, {"k": -1}, {"k": 11, "N": 10, "ldx": 10}, {"t": 0.0}, {"t": -1.0}, {"t": float("inf")},
               {"t": float("nan")}, {"t": 1e-39}, {"ldx": 999}):
        assert call(**kw) == SHAPE, kw
    assert call(kind=3) == DTYPE and call(kind=-1) == DTYPE
    assert call(C=17) == UNSUPPORTED and call(k=129) == UNSUPPORTED and call(B=1 << 24) == UNSUPPORTED
    assert call(N=(1 << 30) + 1, ldx=1 << 31) == UNSUPPORTED and call(kind=0, t=2.0) == UNSUPPORTED
    for name in ("x", "tokens"):
        assert call(**{name: 0}) == NULL, name
    assert call(x=0x100008) == ALIGN and call(stats=0x800004) == ALIGN
    if which != "grad":
        assert call(logprob=0) == NULL and call(ws=0) == NULL and call(ws=0xA00008) == ALIGN and call(bytes=0, B=100) == WORKSPACE
    if which == "forward":
        assert call(k=3, top_ids=0) == NULL and call(k=3, top=0) == NULL
    if which == "step":
        assert call(k=1) == UNSUPPORTED
    if which != "forward":
        assert call(kind=0) == UNSUPPORTED
        assert call(t=2.0 ** -41) == UNSUPPORTED
        assert call(dx=0) == NULL and call(ldd=999) == SHAPE and call(dx=0x900004) == ALIGN
        assert call(dx=0x100000, ldd=1008) == SHAPE                     # x itself, but other strides
        assert call(dx=0x100010) == SHAPE                               # overlaps x
        assert call(B=1 << 22, dx=1 << 50) == UNSUPPORTED               # more workgroups than a launch has
        assert call(B=1 << 20, N=1 << 18, ldx=1 << 18, ldd=1 << 18, dx=1 << 50) == UNSUPPORTED
    if which == "grad":
        assert call(stats=0) == NULL


def test_logprobs_workspace(rdk):
    L, need = rdk.lib(), ctypes.c_size_t()
    d = rdk.LogprobsDesc(B=8, N=128256, C=1, k=5, temperature=1.0)
    for kind in (0, 1, 2):
        assert L.rdk_logprobs_workspace_bytes(ctypes.byref(d), kind, ctypes.byref(need)) == 0 and need.value >= 256
    assert L.rdk_logprobs_workspace_bytes(ctypes.byref(d), 2, None) == NULL
    assert L.rdk_logprobs_workspace_bytes(None, 2, ctypes.byref(need)) == NULL
    assert L.rdk_logprobs_workspace_bytes(ctypes.byref(d), 5, ctypes.byref(need)) == DTYPE
    for B in (1, 8, 1000, (1 << 24) - 1):                               # no size overflows
        big = rdk.LogprobsDesc(B=B, N=1 << 30, C=16, k=0, temperature=1.0)
        assert L.rdk_logprobs_workspace_bytes(ctypes.byref(big), 2, ctypes.byref(need)) == 0 and need.value >= 16 * B


def embed_call(rdk, which, B=4, V=100, d=64, scale=1.0, tt=1, rt=2, ldt=64, ldo=64, accumulate=0, bytes=1 << 40, **at):
    L = rdk.lib()
    p = {name: 0x100000 * (i + 1) for i, name in enumerate(("ids", "table", "rows", "ws"))}
    p.update(at)
    q = {name: vp(a) for name, a in p.items()}
    desc = rdk.EmbedDesc(B=B, V=V, d=d, scale=scale)
    if which == "forward":
        return L.rdk_embed(ctypes.byref(desc), None, q["ids"], q["table"], tt, ldt, q["rows"], rt, ldo, None)
    return L.rdk_embed_grad(ctypes.byref(desc), None, q["ids"], q["rows"], rt, ldo, q["table"], tt, ldt, accumulate, q["ws"], bytes, None)


@pytest.mark.parametrize("which", ["forward", "grad"])
def test_embed_refusals(rdk, which):
    call = lambda **kw: embed_call(rdk, which, **kw)  # noqa: E731
    for kw in ({"B": 0}, {"V": 0}, {"d": 0}, {"d": -1}, {"scale": float("inf")}, {"scale": float("nan")}, {"ldt": 63}, {"ldo": 63}, {"ldt": 1 << 40},
               {"table": 0x300000 - 64}, {"rows": 0x200010}):
        assert call(**kw) == SHAPE, kw
    assert call(B=1 << 24) == UNSUPPORTED and call(V=(1 << 29) + 1) == UNSUPPORTED and call(d=(1 << 20) + 1, ldt=1 << 21, ldo=1 << 21) == UNSUPPORTED
    for kw in ({"tt": 0}, {"tt": 3}, {"rt": 0}, {"rt": -1}):
        assert call(**kw) == DTYPE, kw
    for name in ("ids", "table", "rows") + (("ws",) if which == "grad" else ()):
        assert call(**{name: 0}) == NULL, name
    assert call(table=0x200008) == ALIGN and call(rows=0x300002) == ALIGN
    if which == "grad":
        assert call(ids=0x200100) == SHAPE                              # what is written lies over the ids
        assert call(ws=0x400008) == ALIGN and call(bytes=0, B=5000) == WORKSPACE
    else:
        assert call(ids=0x300040) == SHAPE


def test_embed_workspace(rdk):
    L, need = rdk.lib(), ctypes.c_size_t()
    d = rdk.EmbedDesc(B=16384, V=128256, d=2048, scale=1.0)
    assert L.rdk_embed_grad_workspace_bytes(ctypes.byref(d), ctypes.byref(need)) == 0 and need.value >= 8 * 16384
    assert L.rdk_embed_grad_workspace_bytes(ctypes.byref(d), None) == NULL and L.rdk_embed_grad_workspace_bytes(None, ctypes.byref(need)) == NULL
    last = 0
    for B in (1, 1024, 1025, 16384, 16385, 1 << 20, (1 << 24) - 1):
        d = rdk.EmbedDesc(B=B, V=1 << 29, d=64, scale=1.0)
        assert L.rdk_embed_grad_workspace_bytes(ctypes.byref(d), ctypes.byref(need)) == 0 and need.value >= last
        last = need.value


def test_tensors_of_the_host_are_refused(rdk):
    import torch
    x, tokens = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AssertionError):
        rdk.rdk_logprobs(x, tokens)
    with pytest.raises(AssertionError):
        rdk.rdk_logprobs(x, tokens.long())
    with pytest.raises(AssertionError):
        rdk.rdk_embed(tokens, x)
    with pytest.raises(AssertionError):
        rdk.rdk_embed_grad(tokens, x, rdk.EmbedGradOutputs(4, 8, torch.float32, "cpu"))


def test_descriptors_match_the_header(rdk, tmp_path):
    src = tmp_path / "layout.c"
    mirrors = {"rdk_logprobs_desc_t": rdk.LogprobsDesc, "rdk_embed_desc_t": rdk.EmbedDesc}
    lines = ['  printf("%s %%zu\\n", sizeof(%s));' % (t, t) for t in mirrors]
    lines += ['  printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (t, f, t, f) for t, m in mirrors.items() for f, _ in m._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rdk.h"\nint main(void) {\n' + "\n".join(lines) + "\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines():
        key, value = line.rsplit(" ", 1)
        t, _, f = key.partition(".")
        assert (getattr(mirrors[t], f).offset if f else ctypes.sizeof(mirrors[t])) == int(value), key
