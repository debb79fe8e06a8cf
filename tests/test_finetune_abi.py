"""CPU: the C ABI of adapters and distillation (include/finetune/nvfp4_finetune.h) -- what the library exports, the structs'
layout, and the refusals, each of which enqueues nothing."""
import ctypes as C
import re
import subprocess

import pytest
import torch

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import build
from paper_2512_02010_amd import finetune as F

from . import _hip_calls

HEADER = (build.ROOT / "include" / "finetune" / "nvfp4_finetune.h").read_text()
P = 1 << 20           # an aligned address that nothing looks at


def test_exports_are_those_of_the_header():
    declared = re.findall(r"^(?:int|size_t)\s+(nvfp4_\w+)\s*\(", HEADER, flags=re.M)
    assert sorted(declared) == sorted(F.ENTRY_POINTS)
    symbols = subprocess.run(["nm", "-D", "--defined-only", str(B.library_path())], text=True, capture_output=True, check=True).stdout
    assert set(re.findall(r" T (nvfp4_(?!46_)\w+)$", symbols, flags=re.M)) == set(declared)


def test_header_is_plain_c(tmp_path):
    source = tmp_path / "one.c"
    source.write_text('#include "finetune/nvfp4_finetune.h"\n'
                      "_Static_assert(sizeof(nvfp4_adapters_params) == %d, \"\");\n"
                      "_Static_assert(sizeof(nvfp4_distill_params) == %d, \"\");\n" % (C.sizeof(F.AdaptersParams), C.sizeof(F.DistillParams))
                      + "".join("_Static_assert(__builtin_offsetof(%s, %s) == %d, \"\");\n" % (name, f, getattr(cls, f).offset)
                                for name, cls in (("nvfp4_adapters_params", F.AdaptersParams), ("nvfp4_distill_params", F.DistillParams))
                                for f, _ in cls._fields_))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-fsyntax-only", f"-I{build.ROOT / 'include'}", str(source)], check=True)


def _adapters(**kw):
    p = dict(tokens=5, inp=64, out=32, adapters=3, rank=8, ld_x=64, ld_base=32, ld_out=32, ld_dy=32, out_dtype=0)
    p.update(kw)
    return F.AdaptersParams(*(p[f] for f, _ in F.AdaptersParams._fields_))


def _forward(p, room=1 << 30, **kw):
    v = dict(x=P, base=P, a=P, b=P, which=P, scales=P, h=None, out=2 * P, workspace=P)
    v.update(kw)
    return F.lib().nvfp4_adapters_forward(v["x"], C.byref(p) if p else None, v["base"], v["a"], v["b"], v["which"], v["scales"], v["h"],
                                          v["out"], v["workspace"], room, None)


def _backward(p, room=1 << 30, **kw):
    v = dict(dy=P, x=P, h=P, a=P, b=P, which=P, scales=P, dx_base=P, dx=2 * P, da=P, db=P, workspace=P)
    v.update(kw)
    return F.lib().nvfp4_adapters_backward(v["dy"], C.byref(p) if p else None, v["x"], v["h"], v["a"], v["b"], v["which"], v["scales"],
                                           v["dx_base"], v["dx"], v["da"], v["db"], v["workspace"], room, None)


def test_refusals_of_the_adapters():
    back = dict(ld_base=64, ld_out=64)
    for call, names, more in ((_forward, ("x", "a", "b", "which", "scales", "out", "workspace"), {}),
                              (_backward, ("dy", "x", "h", "a", "b", "which", "scales", "da", "db", "workspace"), back)):
        assert call(None) == 1
        for name in names:
            assert call(_adapters(**more), **{name: None}) == 1, name
        for bad in (dict(tokens=-1), dict(tokens=1 << 24), dict(inp=0), dict(inp=60), dict(out=36), dict(out=-8), dict(adapters=0),
                    dict(adapters=2049), dict(rank=0), dict(rank=129), dict(ld_x=56), dict(ld_x=1 << 41), dict(ld_out=24),
                    dict(ld_base=24), dict(inp=(1 << 22) + 8, ld_x=1 << 23), dict(out=(1 << 22) + 8)):
            assert call(_adapters(**{**more, **bad})) == 2, bad
        for bad in (dict(ld_x=68), dict(ld_base=68), dict(ld_out=68)):
            assert call(_adapters(**{**more, **bad})) == 3, bad
        for name in names:
            if name not in ("which", "scales", "h"):
                assert call(_adapters(**more), **{name: P + 8}) == 3, name
            else:
                assert call(_adapters(**more), **{name: P + 2}) == 3, name
        need = F.lib().nvfp4_adapters_workspace_bytes(C.byref(_adapters(**more)), int(call is _backward))
        assert need > 0 and call(_adapters(**more), room=need - 1) == 4
    assert _backward(_adapters(ld_base=64, ld_out=64, ld_dy=16)) == 2
    assert _backward(_adapters(ld_base=64, ld_out=64, ld_dy=36)) == 3
    assert _forward(_adapters(out_dtype=2)) == 4
    # rows times stride past 64 bits
    assert _forward(_adapters(tokens=(1 << 24) - 1, ld_x=1 << 40)) == 2 and _forward(_adapters(tokens=(1 << 24) - 1, ld_out=1 << 40)) == 2
    # in place, but with another stride
    assert _forward(_adapters(ld_out=40), base=P, out=P) == 2 and _backward(_adapters(ld_base=64, ld_out=72), dx_base=P, dx=P) == 2
    assert _forward(_adapters(), h=P + 2) == 3 and _forward(_adapters(), base=P + 4) == 3
    assert _backward(_adapters(**back), dx=P + 4) == 3 and _backward(_adapters(**back), dx_base=P + 4) == 3
    for p in (None, _adapters(rank=0), _adapters(inp=12), _adapters(tokens=-1)):
        assert F.lib().nvfp4_adapters_workspace_bytes(C.byref(p) if p else None, 0) == 0
    with pytest.raises(B.Nvfp4Error):
        F.adapters_workspace(16, 60, 64, 1, 8, False, device="cpu")


def _distill(**kw):
    p = dict(rows=4, vocab=101, ld=101, top=8, temperature=1.0, x_dtype=0, teacher_dtype=1, index_dtype=0)
    p.update(kw)
    return F.DistillParams(*(p[f] for f, _ in F.DistillParams._fields_))


def _distill_calls():
    lib = F.lib()

    def forward(p, logits=P, teacher=P, index=P, loss=P, lse=P):
        return lib.nvfp4_distill_forward(logits, C.byref(p) if p else None, teacher, index, loss, lse, None)

    def backward(p, logits=P, teacher=P, index=P, lse=P, weight=P, dlogits=P):
        return lib.nvfp4_distill_backward(logits, C.byref(p) if p else None, teacher, index, lse, weight, dlogits, None)

    def step(p, logits=P, teacher=P, index=P, weight=P, loss=P, dlogits=P):
        return lib.nvfp4_distill_step(logits, C.byref(p) if p else None, teacher, index, weight, loss, dlogits, None)

    return ((forward, ("logits", "teacher", "index", "loss")), (backward, ("logits", "teacher", "index", "lse", "dlogits")),
            (step, ("logits", "teacher", "index", "loss", "dlogits")))


def test_refusals_of_the_distillation():
    for call, names in _distill_calls():
        assert call(None) == 1
        for name in names:
            assert call(_distill(), **{name: None}) == 1, name
            assert call(_distill(), **{name: P + 1}) == 3, name
        for bad in (dict(rows=-1), dict(rows=(1 << 21) + 1), dict(vocab=0), dict(vocab=1 << 31, ld=1 << 31), dict(ld=100), dict(top=0),
                    dict(top=1025), dict(rows=1 << 20, ld=1 << 21)):
            assert call(_distill(**bad)) == 2, bad
        for bad in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")),
                    dict(x_dtype=2), dict(teacher_dtype=2), dict(index_dtype=2)):
            assert call(_distill(**bad)) == 4, bad
        assert call(_distill(x_dtype=1), logits=P + 2) == 3
        assert call(_distill(), teacher=P + 2) == 3 and call(_distill(index_dtype=1), index=P + 4) == 3
        if "dlogits" in names:                       # rows that begin at other places of a 16-byte piece
            assert call(_distill(), dlogits=P + 2) == 3
            assert call(_distill(), weight=P + 2) == 3


def test_refused_calls_and_calls_without_rows_make_no_hip_call():
    made = _hip_calls.run("""
from paper_2512_02010_amd import finetune as F
lib = F.lib()
ok = F.AdaptersParams(0, 64, 32, 3, 8, 64, 32, 32, 32, 0)
bad = F.AdaptersParams(4, 60, 32, 3, 8, 64, 32, 32, 32, 0)
assert lib.nvfp4_adapters_forward(None, C.byref(ok), None, P, P, None, P, None, None, P, 1 << 20, None) == 0
assert lib.nvfp4_adapters_forward(P, C.byref(bad), P, P, P, P, P, None, P, P, 1 << 20, None) == 2
assert lib.nvfp4_adapters_backward(P, C.byref(bad), P, P, P, P, P, P, P, P, P, P, P, 1 << 20, None) == 2
d, none = F.DistillParams(4, 0, 8, 8, 1.0, 0, 1, 0), F.DistillParams(0, 8, 8, 8, 1.0, 0, 1, 0)
assert lib.nvfp4_distill_forward(P, C.byref(d), P, P, P, P, None) == 2
assert lib.nvfp4_distill_forward(None, C.byref(none), None, None, None, None, None) == 0
assert lib.nvfp4_distill_backward(None, C.byref(none), None, None, None, None, None, None) == 0
assert lib.nvfp4_distill_step(None, C.byref(none), None, None, None, None, None, None) == 0
result = calls()
""")
    assert made == []


def test_python_refuses_tensors_that_do_not_fit():
    """Whatever is no device tensor is refused before the library is called."""
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    a, b = torch.zeros((2, 8, 64), dtype=torch.bfloat16), torch.zeros((2, 32, 8), dtype=torch.bfloat16)
    which, scales, h = torch.zeros(4, dtype=torch.int32), torch.ones(2), torch.zeros((4, 8))
    with pytest.raises(AssertionError, match="device tensor"):
        F.nvfp4_adapters_forward(x, None, a, b, which, scales)
    with pytest.raises(AssertionError, match="must be a tensor"):
        F.nvfp4_adapters_forward(None, None, a, b, which, scales)
    with pytest.raises(AssertionError, match="device tensor"):
        F.nvfp4_adapters_backward(x[:, :32], x, h, a, b, which, scales)
    for call in (F.nvfp4_distill_forward, F.nvfp4_distill_step):
        with pytest.raises(AssertionError, match="device tensor"):
            call(x, torch.zeros((4, 2)), torch.zeros((4, 2), dtype=torch.int32))
    with pytest.raises(AssertionError, match="device tensor"):
        F.nvfp4_distill_backward(x, torch.zeros((4, 2)), torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4))
