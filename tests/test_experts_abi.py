"""CPU: the C ABI of the products with unquantized activations and of the routing of tokens (include/finetune/nvfp4_finetune.h): the
structs' layout, the refusals, each of which enqueues nothing, and what an accepted call asks of the HIP runtime."""
import ctypes as C
import subprocess

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2512_02010_amd import binding as B
from paper_2512_02010_amd import build
from paper_2512_02010_amd import experts as X
from paper_2512_02010_amd import finetune as F

from . import _hip_calls
from .test_finetune_host import _report

P = 1 << 20           # an aligned address that nothing looks at


def test_structs_are_those_of_the_header(tmp_path):
    source = tmp_path / "one.c"
    source.write_text('#include "finetune/nvfp4_finetune.h"\n' + "".join(
        "_Static_assert(sizeof(%s) == %d, \"\");\n" % (name, C.sizeof(cls))
        + "".join("_Static_assert(__builtin_offsetof(%s, %s) == %d, \"\");\n" % (name, f, getattr(cls, f).offset) for f, _ in cls._fields_)
        for name, cls in (("nvfp4_product_params", F.ProductParams), ("nvfp4_experts_params", F.ExpertsParams))))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-fsyntax-only", f"-I{build.ROOT / 'include'}", str(source)], check=True)


def _product(**kw):
    p = dict(rows=5, inp=64, out=32, experts=1, slots=5, ld_x=64, ld_out=32, x_dtype=0, out_dtype=0, flags=0)
    p.update(kw)
    return F.ProductParams(*(p[f] for f, _ in F.ProductParams._fields_))


def _weight(p, **kw):
    v = dict(x=P, codes=P, scales=P, alpha=P, out=P)
    v.update(kw)
    return F.lib().nvfp4_weight_product(v["x"], C.byref(p) if p else None, v["codes"], v["scales"], v["alpha"], v["out"], None)


def _experts(p, **kw):
    v = dict(x=P, token=P, begin=P, codes=P, scales=P, alpha=P, out=P)
    v.update(kw)
    return F.lib().nvfp4_experts_product(v["x"], C.byref(p) if p else None, v["token"], v["begin"], v["codes"], v["scales"], v["alpha"],
                                         v["out"], None)


def test_refusals_of_the_products():
    for call, names in ((_weight, ("x", "codes", "scales", "alpha", "out")), (_experts, ("x", "begin", "codes", "scales", "alpha", "out"))):
        assert call(None) == 1
        for name in names:
            assert call(_product(), **{name: None}) == 1, name
            assert call(_product(), **{name: P + (2 if name in ("alpha", "begin") else 8)}) == 3, name
        for bad in (dict(rows=-1), dict(rows=1 << 24), dict(inp=0), dict(inp=48), dict(inp=(1 << 22) + 32, ld_x=1 << 23), dict(out=0),
                    dict(out=(1 << 22) + 1, ld_out=1 << 23), dict(experts=0), dict(experts=1025), dict(slots=-1), dict(slots=(1 << 30) + 1),
                    dict(ld_x=56), dict(ld_out=31), dict(ld_x=1 << 40), dict(ld_out=1 << 40), dict(flags=B.GEMM_B_TILE_SCALES, out=40, ld_out=40)):
            assert call(_product(**bad), **({} if call is _weight else dict(token=P))) == 2, bad
        assert call(_product(ld_x=68)) == 3
        for bad in (dict(x_dtype=2), dict(out_dtype=2), dict(flags=1), dict(flags=4)):
            assert call(_product(**bad)) == 4, bad
        # sizes before pointers that what has no element may well lack
        assert call(_product(rows=-1), **dict.fromkeys(names)) == 2
    assert _weight(_product(experts=2)) == 2 and _weight(_product(slots=4)) == 2
    assert _experts(_product(slots=4), token=None) == 2 and _experts(_product(), token=P + 2) == 3
    # rows of x times their stride past 64 bits
    assert _weight(_product(rows=(1 << 24) - 1, slots=(1 << 24) - 1, ld_x=1 << 40)) == 2


def _routing(**kw):
    p = dict(tokens=5, top=2, experts=4, width=64, ld_token=64, ld_base=64, ld_slot=64, ld_dslot=64, token_dtype=0, slot_dtype=0, index_dtype=0)
    p.update(kw)
    return F.ExpertsParams(*(p[f] for f, _ in F.ExpertsParams._fields_))


def _sort(p, room=1 << 30, **kw):
    v = dict(ids=P, place=P, token=P, begin=P, workspace=P)
    v.update(kw)
    return F.lib().nvfp4_experts_sort(v["ids"], C.byref(p) if p else None, v["place"], v["token"], v["begin"], v["workspace"], room, None)


def _spread(p, **kw):
    v = dict(x=P, place=P, xs=P)
    v.update(kw)
    return F.lib().nvfp4_experts_spread(v["x"], C.byref(p) if p else None, v["place"], v["xs"], None)


def _combine(p, **kw):
    v = dict(ys=P, place=P, weights=P, base=P, y=2 * P)
    v.update(kw)
    return F.lib().nvfp4_experts_combine(v["ys"], C.byref(p) if p else None, v["place"], v["weights"], v["base"], v["y"], None)


def _backward(p, **kw):
    v = dict(dy=P, ys=P, place=P, weights=P, dys=2 * P, dweights=P)
    v.update(kw)
    return F.lib().nvfp4_experts_combine_backward(v["dy"], C.byref(p) if p else None, v["ys"], v["place"], v["weights"], v["dys"], v["dweights"],
                                                  None)


def test_refusals_of_the_sort():
    assert _sort(None) == 1
    for name in ("ids", "place", "token", "begin", "workspace"):
        assert _sort(_routing(), **{name: None}) == 1, name
        assert _sort(_routing(), **{name: P + (8 if name == "workspace" else 2)}) == 3, name
    assert _sort(_routing(index_dtype=1), ids=P + 4) == 3
    for bad in (dict(tokens=-1), dict(tokens=1 << 24), dict(top=0), dict(top=65), dict(experts=0), dict(experts=1025), dict(tokens=(1 << 24) - 1, top=64 + 1)):
        assert _sort(_routing(**bad)) == 2, bad
        assert F.lib().nvfp4_experts_workspace_bytes(C.byref(_routing(**bad))) == 0
    assert _sort(_routing(index_dtype=2)) == 4
    for sizes in (dict(), dict(tokens=5000, top=8, experts=100), dict(tokens=(1 << 24) - 1, top=64, experts=1024)):
        need = F.lib().nvfp4_experts_workspace_bytes(C.byref(_routing(**sizes)))
        assert 16 <= need <= 1 << 20 and _sort(_routing(**sizes), room=need - 1) == 4
    assert F.lib().nvfp4_experts_workspace_bytes(None) == 0
    with pytest.raises(B.Nvfp4Error):
        X.experts_workspace(10, 65, 4, device="cpu")


def test_refusals_of_the_rows():
    for call, names, strides in ((_spread, ("x", "place", "xs"), ("ld_token", "ld_slot")), (_combine, ("ys", "place", "y"), ("ld_token", "ld_slot", "ld_base")),
                                 (_backward, ("dy", "ys", "place", "weights", "dys", "dweights"), ("ld_token", "ld_slot", "ld_dslot"))):
        assert call(None) == 1
        for name in names:
            assert call(_routing(), **{name: None}) == 1, name
            assert call(_routing(), **{name: P + (2 if name in ("place", "weights", "dweights") else 8)}) == 3, name
        for bad in (dict(tokens=-1), dict(tokens=1 << 24), dict(top=0), dict(top=65), dict(width=0), dict(width=60), dict(width=(1 << 22) + 8),
                    *({s: 56} for s in strides), *({s: 1 << 40} for s in strides)):
            assert call(_routing(**bad)) == 2, bad
        for s in strides:
            assert call(_routing(**{s: 68})) == 3, s
        for bad in (dict(token_dtype=2), dict(slot_dtype=2)):
            assert call(_routing(**bad)) == 4, bad
        assert call(_routing(tokens=0), **dict.fromkeys(names)) == 0
    assert _combine(_routing(), weights=P + 2) == 3 and _combine(_routing(), base=P + 8) == 3
    # in place, but with another stride
    assert _combine(_routing(ld_token=72), base=P, y=P) == 2 and _backward(_routing(ld_dslot=72), ys=P, dys=P) == 2


def test_launches_of_a_call():
    """One for every call, two for a sort of more than 4096 pairs; none for a call that is refused or has no rows."""
    made = _hip_calls.run("""
from paper_2512_02010_amd import finetune as F
lib, result = F.lib(), {}
def kinds():
    return [c[0] for c in calls()]
for T, k, E in ((0, 2, 8), (5, 2, 8), (2048, 2, 1024), (2049, 2, 8), (100000, 8, 1024)):
    p = F.ExpertsParams(T, k, E, 64, 64, 64, 64, 64, 0, 0, 0)
    assert lib.nvfp4_experts_sort(P, C.byref(p), P, P, P, P, 1 << 30, None) == 0
    result[f"sort {T * k}"] = kinds()
    assert lib.nvfp4_experts_spread(P, C.byref(p), P, 2 * P, None) == 0
    assert lib.nvfp4_experts_combine(P, C.byref(p), P, P, P, 2 * P, None) == 0
    assert lib.nvfp4_experts_combine_backward(P, C.byref(p), P, P, P, 2 * P, P, None) == 0
    result[f"rows {T}"] = kinds()
bad = F.ProductParams(5, 48, 64, 1, 5, 64, 64, 0, 0, 0)
none = F.ProductParams(0, 64, 64, 1, 0, 64, 64, 0, 0, 0)
assert lib.nvfp4_weight_product(P, C.byref(bad), P, P, P, P, None) == 2
assert lib.nvfp4_weight_product(None, C.byref(none), P, P, P, None, None) == 0
assert lib.nvfp4_experts_product(None, C.byref(none), None, P, P, P, P, None, None) == 0
result["none"] = kinds()
for T in (1, 10, 100, 1000, 5000):
    for dtype in (0, 1):
        p = F.ProductParams(T, 512, 1000, 3, T, 512, 1000, dtype, 0, 0)
        assert lib.nvfp4_experts_product(P, C.byref(p), P, P, P, P, P, P, None) == 0
        result[f"product {T} {dtype}"] = [k for k in kinds() if k != "set_attribute"]
""")
    for name, kinds in made.items():
        what, n = (name.split() + ["0"])[:2]
        launches = [k for k in kinds if k != "set_attribute"]
        want = {"sort": 2 if int(n) > 4096 else 1, "rows": 0 if n == "0" else 3, "product": 1, "none": 0}[what]
        assert launches == ["launch"] * want, (name, kinds)
        if what == "none":
            assert kinds == []


def test_no_kernel_spills():
    """The products count their copies by hand: a spill would add memory instructions of the compiler's own to the counts."""
    for source, least in (("weight_product.hip", 52), ("experts.hip", 42)):
        kernels = {k: v for k, v in _report(source).items() if "LDS" in v}
        assert len(kernels) >= least, (source, len(kernels))
        spilled = {k: v["ScratchSize"] for k, v in kernels.items() if v["ScratchSize"]}
        assert not spilled, spilled


def test_python_refuses_tensors_that_do_not_fit():
    x, codes, scales, alpha = torch.zeros((4, 64)), torch.zeros((32, 32), dtype=torch.uint8), torch.zeros((32, 4), dtype=torch.uint8), torch.ones(1)
    place, ids = torch.zeros((4, 2), dtype=torch.int32), torch.zeros((4, 2), dtype=torch.int64)
    for call in (lambda: X.nvfp4_weight_product(x, codes, scales, alpha), lambda: X.nvfp4_experts_product(x, ids, codes, scales, alpha),
                 lambda: X.nvfp4_experts_sort(ids, 4), lambda: X.nvfp4_experts_spread(x, place), lambda: X.nvfp4_experts_combine(x, place),
                 lambda: X.nvfp4_experts_combine_backward(x, x, place, alpha)):
        with pytest.raises(AssertionError, match="device tensor"):
            call()


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
def test_python_refuses_what_lies_elsewhere_or_is_of_another_kind():
    """(Tensors without memory stand for those of two devices.)"""
    mode = FakeTensorMode()
    with mode:
        def zeros(*shape, dtype=torch.bfloat16, device="cuda:0"):
            return torch.empty(shape, dtype=dtype, device=device)

        i32, f32, u8 = torch.int32, torch.float32, torch.uint8
        x, codes, scales, alpha = zeros(4, 64), zeros(32, 32, dtype=u8), zeros(32, 4, dtype=u8), zeros(1, dtype=f32)
        three = dict(codes=zeros(3, 32, 32, dtype=u8), scales=zeros(3, 32, 4, dtype=u8), alpha=zeros(3, dtype=f32))
        begin, place, ids, weights = zeros(4, dtype=i32), zeros(4, 2, dtype=i32), zeros(4, 2, dtype=i32), zeros(4, 2, dtype=f32)
        xs, apart = zeros(8, 64), torch.empty_strided((4, 64), (1, 4), dtype=torch.bfloat16, device="cuda:0")
        wrong = [
            (lambda: X.nvfp4_weight_product(x, zeros(32, 32, dtype=u8, device="cuda:1"), scales, alpha), "codes must be on the device"),
            (lambda: X.nvfp4_weight_product(x, zeros(32, 16, dtype=u8), scales, alpha), "codes must be of a shape"),
            (lambda: X.nvfp4_weight_product(x, codes, scales, alpha, flags=B.GEMM_B_TILE_SCALES), "scales must be of a shape"),
            (lambda: X.nvfp4_weight_product(zeros(4, 64, dtype=torch.float16), codes, scales, alpha), "x must be BF16 or fp32"),
            (lambda: X.nvfp4_weight_product(x, codes, scales, alpha, out=zeros(4, 32, dtype=torch.float16)), "out must be BF16 or fp32"),
            (lambda: X.nvfp4_weight_product(x, codes, scales, alpha, out_dtype=2), "out_dtype"),
            (lambda: X.nvfp4_weight_product(apart, codes, scales, alpha), "adjacent columns"),
            (lambda: X.nvfp4_experts_product(x, zeros(3, dtype=i32), **three), "begin must be of a shape"),
            (lambda: X.nvfp4_experts_product(x, begin, **three, token=zeros(6, dtype=torch.int64)), "token must be Int"),
            (lambda: X.nvfp4_experts_sort(weights, 4), "ids must be int32 or int64"),
            (lambda: X.nvfp4_experts_sort(ids, 4, workspace=zeros(1 << 16, dtype=u8, device="cuda:1")), "workspace must be on the device"),
            (lambda: X.nvfp4_experts_spread(zeros(5, 64), place), "x must be of a shape"),
            (lambda: X.nvfp4_experts_combine(x, place), "ys must be of a shape"),
            (lambda: X.nvfp4_experts_combine(xs, place, weights=zeros(4, 3, dtype=f32)), "weights must be of a shape"),
        ]
    for call, text in wrong:
        with mode, pytest.raises(AssertionError, match=text):
            call()
    with pytest.raises(B.Nvfp4Error):
        X.nvfp4_experts_sort(ids, 1025)
