"""What root-mean-square norm, cross entropy and AdamW refuse, on the host, before anything is launched; their structs and scratch sizes."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2110_08450_amd import binding as smfg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x7f0000001000  # never dereferenced: every call below is refused first
F32, F16, BF16, I8, E4M3 = 0, 1, 2, 3, 4
NULL, ARG, ROOM = smfg.ERR_NULL_PTR, smfg.ERR_INVALID_ARG, smfg.ERR_CAPACITY

RMS = dict(x=P, xstride=64, dtype=F16, residual=P + 4096, rstride=64, total=P + 8192, tstride=64, num=P, max_rows=4, dim=40, w=P, ptype=F32, eps=1e-5,
           y=P + 12288, ystride=64, ytype=F16, scales=None, sstride=0, group=0, rstd=P, stream=None)
BYTES = dict(RMS, ytype=E4M3, scales=P, sstride=2, group=32)
RGRAD = dict(dy=P, dstride=8, t=P + 4096, tstride=8, dtype=F16, dtotal=P + 12288, dtstride=8, num=P, max_rows=4, dim=8, w=P, ptype=F32, rstd=P, dx=P + 8192,
             dxstride=8, dw=P, scratch=P, bytes=1 << 40, stream=None)
LOSS = dict(x=P, xstride=8, dtype=BF16, labels=P, label_bytes=8, num=P, max_rows=4, classes=8, reduction=0, scale=1.0, loss=P, row_loss=P, dx=P + 4096, dxstride=8,
            scratch=P, bytes=1 << 40, stream=None)


def call(name, good, **change):
    args = dict(good)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(smfg.lib(), name)(*args.values())


@pytest.mark.parametrize("name,good,change,code", [
    *[("smfg_rms_norm", RMS, {k: None}, NULL) for k in ("x", "num", "y")],
    ("smfg_rms_norm", BYTES, dict(scales=None), NULL),
    *[("smfg_rms_norm", RMS, c, ARG) for c in (
        dict(dim=0), dict(dim=(1 << 23) + 1), dict(max_rows=-1), dict(max_rows=1 << 31), dict(xstride=39), dict(rstride=39), dict(tstride=39), dict(ystride=39),
        dict(dtype=3), dict(dtype=4), dict(ptype=BF16), dict(ptype=3), dict(eps=-1.0), dict(eps=float("nan")), dict(x=P + 1), dict(residual=P + 1),
        dict(total=P + 1), dict(y=P + 1), dict(w=P + 2), dict(rstd=P + 2), dict(num=P + 4), dict(ytype=F32), dict(ytype=5), dict(scales=P), dict(group=32),
        dict(residual=None),  # a sum of nothing
        dict(y=P, ystride=72), dict(y=P + 4096, ystride=72), dict(total=P, tstride=72), dict(total=P + 4096, tstride=72), dict(total=P + 12288))],
    *[("smfg_rms_norm", BYTES, c, ARG) for c in (
        dict(group=16), dict(group=-32), dict(group=256), dict(group=48), dict(sstride=1), dict(sstride=0, group=0), dict(scales=P + 2), dict(ystride=39),
        dict(ytype=I8, y=P), dict(y=P + 4096), dict(sstride=1 << 40))],
    *[("smfg_rms_norm_grad", RGRAD, {k: None}, NULL) for k in ("dy", "t", "num", "rstd", "scratch")],
    *[("smfg_rms_norm_grad", RGRAD, c, ARG) for c in (
        dict(dim=0), dict(max_rows=-1), dict(max_rows=1 << 31), dict(dstride=7), dict(tstride=7), dict(dtstride=7), dict(dxstride=7), dict(dtype=5), dict(ptype=BF16),
        dict(dy=P + 1), dict(t=P + 1), dict(dtotal=P + 1), dict(dx=P + 1), dict(w=P + 2), dict(dw=P + 1), dict(rstd=P + 2), dict(num=P + 4), dict(scratch=P + 8),
        dict(dx=P, dxstride=16), dict(dx=P + 4096, dxstride=9), dict(dx=P + 12288, dxstride=9))],
    ("smfg_rms_norm_grad", RGRAD, dict(bytes=64), ROOM),
    *[("smfg_cross_entropy", LOSS, {k: None}, NULL) for k in ("x", "labels", "num", "loss", "scratch")],
    *[("smfg_cross_entropy", LOSS, c, ARG) for c in (
        dict(classes=0), dict(classes=(1 << 23) + 1), dict(max_rows=-1), dict(max_rows=1 << 31), dict(xstride=7), dict(dxstride=7), dict(dtype=3), dict(label_bytes=2),
        dict(reduction=2), dict(reduction=-1), dict(scale=float("inf")), dict(scale=float("nan")), dict(x=P + 1), dict(labels=P + 4), dict(num=P + 4), dict(loss=P + 2),
        dict(row_loss=P + 1), dict(dx=P + 1), dict(dx=P, dxstride=16), dict(scratch=P + 64))],
    ("smfg_cross_entropy", LOSS, dict(bytes=64), ROOM)])
def test_refusals(name, good, change, code):
    assert call(name, good, **change) == code


def test_nothing_to_do_is_not_refused():
    assert call("smfg_rms_norm", RMS, max_rows=0, x=None, y=None) == smfg.OK
    assert call("smfg_rms_norm", BYTES, max_rows=0, x=None, y=None, scales=None) == smfg.OK
    assert call("smfg_rms_norm_grad", RGRAD, max_rows=0, t=None, dy=None, rstd=None, dw=None, scratch=None) == smfg.OK
    assert call("smfg_rms_norm_grad", RGRAD, dx=None, dw=None, scratch=None) == smfg.OK
    assert smfg.lib().smfg_adamw((smfg._Param * 1)(), 0, hyper(), None) == smfg.OK
    assert adamw(numel=0, param=None, grad=None, m=None, v=None) == smfg.OK
    assert smfg.lib().smfg_adamw_values(None, None, 0, 0, 0, None, F32, None) == smfg.OK


def hyper(**change):
    h = smfg._AdamW(1e-3, 0.9, 0.999, 1e-8, 1.0, float("inf"), 1, None, None, None)
    for k, v in change.items():
        setattr(h, k, v)
    return h


def param(**change):
    p = smfg._Param(P, P, P, P, None, None, None, 4096, F32, F16, 0, 32, 0.01, 0, None, None, 0)
    for k, v in change.items():
        setattr(p, k, v)
    return (smfg._Param * 1)(p)


def adamw(h=None, n=1, **change):
    return smfg.lib().smfg_adamw(param(**change), n, h if h is not None else hyper(), None)


@pytest.mark.parametrize("change", [
    dict(numel=-1), dict(numel=1 << 48), dict(param_dtype=3), dict(grad_dtype=3), dict(param_dtype=F16, grad_dtype=BF16), dict(param_dtype=BF16, grad_dtype=F16),
    dict(state_bits=16), dict(state_bits=0), dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(weight_decay=float("inf")), dict(copy=P, copy_dtype=F32),
    dict(copy=P, copy_dtype=3), dict(copy=P + 1, copy_dtype=F16), dict(copy=P, copy_dtype=F16, param_dtype=F16), dict(row_elems=-1), dict(row_elems=100),
    dict(row_elems=(1 << 23) + 1), dict(d_rows=P), dict(d_row_ids=P, num_rows=10), dict(d_row_ids=P, row_elems=64), dict(d_row_ids=P, row_elems=64, num_rows=1 << 31),
    dict(d_row_ids=P + 2, row_elems=64, num_rows=10), dict(d_rows=P + 4, row_elems=64), dict(param=P + 2), dict(grad=P + 1), dict(m=P + 2), dict(v=P + 1),
    dict(state_bits=8, m_scale=P + 2, v_scale=P), dict(state_bits=8, m_scale=P, v_scale=P + 1), dict(numel=1 << 33, row_elems=2)])
def test_adamw_refuses_tensors(change):
    assert adamw(**change) == ARG


def test_adamw_refusals():
    L = smfg.lib()
    for k in ("param", "grad", "m", "v"):
        assert adamw(**{k: None}) == NULL
    assert adamw(state_bits=8, m_scale=P) == NULL and adamw(state_bits=8, v_scale=P) == NULL
    assert L.smfg_adamw(None, 1, hyper(), None) == NULL and L.smfg_adamw(param(), 1, None, None) == NULL
    assert L.smfg_adamw(param(), -1, hyper(), None) == ARG
    inf, nan = float("inf"), float("nan")
    for bad in (dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta1=nan), dict(beta2=1.0), dict(beta2=-1e-9), dict(eps=-1e-9), dict(eps=0.0), dict(eps=1e-39), dict(eps=1e39), dict(eps=inf),
                dict(eps=nan), dict(scale=inf), dict(scale=nan), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=nan), dict(step=0), dict(step=-1),
                dict(step=1 << 48), dict(step=-1, d_step=P), dict(d_step=P + 4), dict(d_lr=P + 2), dict(d_norm=P + 1)):
        assert adamw(hyper(**bad)) == ARG, bad
    huge = (smfg._Param * 70_000)(*[param(numel=(1 << 48) - 1, grad_dtype=F32)[0]] * 70_000)
    assert L.smfg_adamw(huge, 70_000, hyper(), None) == ARG  # more blocks than have numbers


VALUES = dict(codes=P, scales=P, numel=4096, row_elems=0, second=0, out=P, otype=F32, stream=None)


@pytest.mark.parametrize("change,code", [*[({k: None}, NULL) for k in ("codes", "scales", "out")],
                                         *[(c, ARG) for c in (dict(numel=-1), dict(numel=1 << 48), dict(row_elems=-1), dict(row_elems=100), dict(row_elems=1 << 24),
                                                              dict(second=2), dict(otype=3), dict(scales=P + 2), dict(out=P + 2), dict(numel=1 << 33, row_elems=2))]])
def test_adamw_values_refusals(change, code):
    assert call("smfg_adamw_values", VALUES, **change) == code


def test_scratch_sizes_are_host_only():
    L = smfg.lib()
    assert L.smfg_rms_norm_grad_scratch_bytes(10, 100) >= 400 and L.smfg_rms_norm_grad_scratch_bytes(0, 100) >= 0
    assert L.smfg_cross_entropy_scratch_bytes(0, 1) > 0 and L.smfg_cross_entropy_scratch_bytes((1 << 31) - 1, 1 << 23) > 0
    for name in ("smfg_rms_norm_grad_scratch_bytes", "smfg_cross_entropy_scratch_bytes"):
        for n, dim in ((-1, 1), (1 << 31, 1), (1, 0), (1, (1 << 23) + 1)):
            assert getattr(L, name)(n, dim) == -1
        for dim in (1, 200, 5000, 40_000):  # scratch has room for calls of fewer rows
            sizes = [getattr(L, name)(n, dim) for n in (0, 1, 7, 100, 5000, 8192, 8193, 10 ** 6, 2 ** 31 - 1)]
            assert sizes == sorted(sizes)
    with pytest.raises(smfg.SmfgError):
        smfg.cross_entropy_workspace(1, 0)
    with pytest.raises(smfg.SmfgError):
        smfg.rms_norm_grad_workspace(-1, 5)


@pytest.mark.parametrize("name,mirror", [("smfg_param_t", smfg._Param), ("smfg_adamw_t", smfg._AdamW)])
def test_struct_layout_matches_the_binding(name, mirror, tmp_path):
    fields = [f for f, _ in mirror._fields_]
    src = tmp_path / "layout.c"
    src.write_text(f'#include "smfg.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {{\n  printf("size %zu\\n", sizeof({name}));\n'
                   + "\n".join(f'  printf("{f} %zu\\n", offsetof({name}, {f}));' for f in fields) + "\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = dict(line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines())
    assert int(got["size"]) == ctypes.sizeof(mirror)
    for f in fields:
        assert int(got[f]) == getattr(mirror, f).offset, f


class OnDevice(torch.Tensor):
    """A tensor on the host that says it is on the device; nothing here is launched."""
    is_cuda = property(lambda self: True)


def tensor(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def test_lists_of_tensors_are_checked():
    """Sizes and types that the binding alone can see."""
    p, g, m, v = [tensor(300) for _ in range(4)]
    smfg.adamw_list([p], [g], [m], [v])
    k, u, s = tensor(300, dtype=torch.int8), tensor(300, dtype=torch.uint8), tensor(3)
    smfg.adamw_list([p], [g], [k], [u], [s], [s.clone()])
    table, states = tensor(4, 200), (tensor(4, 200, dtype=torch.int8), tensor(4, 200, dtype=torch.uint8), tensor(4, 2))
    made = smfg.adamw_list([table], [tensor(3, 200)], [states[0]], [states[1]], [states[2]], [states[2].clone()], rows=[tensor(1, dtype=torch.int64)],
                           row_ids=[tensor(3, dtype=torch.int32)])
    assert made.c[0].row_elems == 200 and made.c[0].num_rows == 4 and made.c[0].numel == 600
    for bad in (dict(g=[tensor(299)]), dict(m=[tensor(301)]), dict(v=[tensor(5)]), dict(m=[k], v=[u]), dict(m=[k], v=[u], m_scales=[tensor(2)], v_scales=[tensor(2)]),
                dict(m=[k], v=[k], m_scales=[s], v_scales=[s]), dict(m=[k], v=[u], m_scales=[s], v_scales=[tensor(4)]), dict(copies=[tensor(10, dtype=torch.float16)]),
                dict(g=[tensor(300, dtype=torch.int32)]), dict(weight_decay=[0.1, 0.2]), dict(m_scales=[s], v_scales=[s])):
        args = dict(p=[p], g=[g], m=[m], v=[v])
        args.update(bad)
        with pytest.raises(AssertionError):
            smfg.adamw_list(args.pop("p"), args.pop("g"), args.pop("m"), args.pop("v"), **args)
    with pytest.raises(AssertionError):
        smfg.adamw_list([p, p], [g, g], [m, tensor(300)], [v, tensor(300)])  # two steps of one tensor at once
    with pytest.raises(AssertionError):
        smfg.adamw_list([table], [tensor(3, 100)], [tensor(4, 200)], [tensor(4, 200)], row_ids=[tensor(3, dtype=torch.int32)])
    with pytest.raises(AssertionError):
        smfg.adamw_list([table], [tensor(3, 200)], [tensor(4, 200)], [tensor(4, 200)], row_ids=[tensor(2, dtype=torch.int32)])


@pytest.mark.parametrize("shared", ["one tensor's scales", "two tensors' m_scales", "two tensors' v_scales", "two tensors' copies"])
def test_lists_refuse_an_output_given_twice(shared):
    """All that a step writes has one place each: of two writers either may be the last."""
    p, g = [tensor(300), tensor(300)], [tensor(300), tensor(300)]
    if shared == "two tensors' copies":
        m, v, copies = [tensor(300), tensor(300)], [tensor(300), tensor(300)], [tensor(300, dtype=torch.float16)] * 2
        lists = dict(copies=copies)
        apart = dict(copies=[copies[0], tensor(300, dtype=torch.float16)])
    else:
        m, v = [tensor(300, dtype=torch.int8) for _ in range(2)], [tensor(300, dtype=torch.uint8) for _ in range(2)]
        a = [tensor(3) for _ in range(4)]
        apart = dict(m_scales=a[:2], v_scales=a[2:])
        lists = {"one tensor's scales": dict(m_scales=a[:2], v_scales=[a[0], a[3]]), "two tensors' m_scales": dict(m_scales=[a[0], a[0]], v_scales=a[2:]),
                 "two tensors' v_scales": dict(m_scales=a[:2], v_scales=[a[2], a[2]])}[shared]
    assert smfg.adamw_list(p, g, m, v, **apart).n == 2
    with pytest.raises(AssertionError, match="twice"):
        smfg.adamw_list(p, g, m, v, **lists)


@pytest.mark.parametrize("by", ["rows", "row_ids"])
def test_scales_of_tensors_that_are_stepped_by_row_have_two_dimensions(by):
    """5 rows of 120 have as many blocks by row as in one piece: 5.  A step by row uses a scale for each row, while one dimension tells adamw_values that the second
    begins at element 128."""
    p, g, m, v = tensor(5, 120), tensor(5, 120), tensor(5, 120, dtype=torch.int8), tensor(5, 120, dtype=torch.uint8)
    more = dict(rows=[tensor(1, dtype=torch.int64)]) if by == "rows" else dict(row_ids=[tensor(5, dtype=torch.int32)])

    def made(*shape, **more):
        return smfg.adamw_list([p], [g], [m], [v], m_scales=[tensor(*shape)], v_scales=[tensor(*shape)], **more)

    assert made(5, 1, **more).c[0].row_elems == 120 == made(5, 1).c[0].row_elems and made(5).c[0].row_elems == 0
    for shape in ((5,), (1, 5), (1, 5, 1), (5, 1, 1), (6, 1)):
        with pytest.raises(AssertionError):
            made(*shape, **more)
    for shape in ((1, 5), (1, 5, 1), (4,), (4, 1)):
        with pytest.raises(AssertionError):
            made(*shape)


@pytest.mark.parametrize("codes,scales", [((5, 120), (1, 5)), ((5, 120), (5, 1, 1)), ((5, 120), (4,)), ((5, 120), (6,)), ((5, 120), (5, 2)), ((600,), (1, 5)), ((600,), (5, 1)),
                                          ((5, 120), ())])
def test_values_refuse_scales_that_are_not_their_rows(codes, scales):
    with pytest.raises(AssertionError):
        smfg.adamw_values(tensor(*codes, dtype=torch.int8), tensor(*scales), tensor(*codes))


def test_a_limit_without_a_norm_is_refused():
    """The norm is found by clip_grad_norm; without one a step would be of the gradients as they are, whatever the limit."""
    empty = smfg.adamw_list([], [], [], [])
    for max_norm in (1.0, 1e30, float("nan")):
        with pytest.raises(AssertionError, match="norm"):
            smfg.adamw(empty, 1, 1e-3, max_norm=max_norm)
