"""What the operators of a training step refuse, on the host, before anything is launched."""
import ctypes
import os
import subprocess

import pytest

from paper_2110_08450_amd import binding as smfg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x7f0000001000  # never dereferenced: every call below is refused first
F32, F16, BF16 = 0, 1, 2
NULL, ARG, ROOM = smfg.ERR_NULL_PTR, smfg.ERR_INVALID_ARG, smfg.ERR_CAPACITY


def call(name, good, **change):
    args = dict(good)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(smfg.lib(), name)(*args.values())


EMBED = dict(table=P, rows=10, tstride=8, ttype=F16, ids=P, id_bytes=4, num=P, max_ids=4, dim=8, scale=1.0, out=P, ostride=8, otype=F16, stream=None)
GRAD = dict(ids=P, id_bytes=8, num=P, max_ids=4, dy=P, dstride=8, dtype=F16, dim=8, scale=1.0, grad=P, rows=10, gstride=8, gtype=F32, accumulate=0,
            scratch=P & ~255, bytes=1 << 40, stream=None)
ROWS = dict(ids=P, id_bytes=8, num=P, max_ids=4, dy=P, dstride=8, dtype=F16, dim=8, scale=1.0, rows=10, row_ids=P, unique=P, grad=P, gstride=8, gtype=F32,
            scratch=P & ~255, bytes=1 << 40, stream=None)
NORM = dict(x=P, xstride=8, dtype=F16, num=P, max_rows=4, dim=8, w=P, b=P, ptype=F32, eps=1e-5, y=P + 4096, ystride=8, mean=P, rstd=P, stream=None)
NGRAD = dict(dy=P, dstride=8, x=P + 4096, xstride=8, dtype=F16, num=P, max_rows=4, dim=8, w=P, ptype=F32, mean=P, rstd=P, dx=P + 8192, dxstride=8, dw=P, db=P,
             scratch=P & ~255, bytes=1 << 40, stream=None)


@pytest.mark.parametrize("name,good,change,code", [
    *[("smfg_embedding", EMBED, {k: None}, NULL) for k in ("table", "ids", "num", "out")],
    *[("smfg_embedding", EMBED, c, ARG) for c in (
        dict(rows=0), dict(rows=1 << 31), dict(tstride=7), dict(ttype=3), dict(id_bytes=2), dict(max_ids=-1), dict(max_ids=1 << 31), dict(dim=0),
        dict(dim=(1 << 23) + 1), dict(ostride=7), dict(otype=F32), dict(otype=BF16), dict(otype=-1), dict(ttype=BF16), dict(table=P + 1), dict(out=P + 1), dict(ids=P + 2),
        dict(num=P + 4))],
    *[("smfg_embedding_grad", GRAD, {k: None}, NULL) for k in ("ids", "num", "dy", "grad", "scratch")],
    *[("smfg_embedding_grad", GRAD, c, ARG) for c in (
        dict(id_bytes=1), dict(max_ids=-1), dict(max_ids=1 << 31), dict(rows=0), dict(rows=1 << 31), dict(dim=0), dict(dstride=7), dict(gstride=1), dict(dtype=3),
        dict(gtype=BF16), dict(dtype=F32, gtype=F16), dict(ids=P + 4), dict(dy=P + 1), dict(grad=P + 2), dict(num=P + 1), dict(scratch=P + 128))],
    ("smfg_embedding_grad", GRAD, dict(bytes=64), ROOM),
    *[("smfg_embedding_grad_rows", ROWS, {k: None}, NULL) for k in ("ids", "num", "dy", "grad", "scratch", "row_ids", "unique")],
    *[("smfg_embedding_grad_rows", ROWS, c, ARG) for c in (dict(row_ids=P + 2), dict(unique=P + 4), dict(rows=0), dict(gstride=7))],
    ("smfg_embedding_grad_rows", ROWS, dict(bytes=64), ROOM),
    *[("smfg_layer_norm", NORM, {k: None}, NULL) for k in ("x", "num", "y")],
    *[("smfg_layer_norm", NORM, c, ARG) for c in (
        dict(dim=0), dict(max_rows=-1), dict(max_rows=1 << 31), dict(xstride=7), dict(ystride=7), dict(dtype=5), dict(ptype=BF16), dict(ptype=9), dict(eps=-1.0),
        dict(eps=float("nan")), dict(x=P + 1), dict(y=P + 1), dict(w=P + 2), dict(b=P + 1), dict(mean=P + 2), dict(rstd=P + 1), dict(num=P + 4),
        dict(y=P, ystride=16))],
    *[("smfg_layer_norm_grad", NGRAD, {k: None}, NULL) for k in ("dy", "x", "num", "mean", "rstd", "scratch")],
    *[("smfg_layer_norm_grad", NGRAD, c, ARG) for c in (
        dict(dim=0), dict(max_rows=-1), dict(dstride=7), dict(xstride=7), dict(dxstride=7), dict(dtype=5), dict(ptype=BF16), dict(dy=P + 1), dict(dx=P + 1),
        dict(w=P + 2), dict(dw=P + 1), dict(db=P + 2), dict(mean=P + 1), dict(rstd=P + 2), dict(num=P + 4), dict(scratch=P + 8), dict(dx=P, dxstride=16),
        dict(dx=P + 4096, dxstride=9))],
    ("smfg_layer_norm_grad", NGRAD, dict(bytes=64), ROOM)])
def test_refusals(name, good, change, code):
    assert call(name, good, **change) == code


def test_nothing_to_do_is_not_refused():
    """No places at all need no arrays of them, and nothing is launched."""
    assert call("smfg_embedding", EMBED, max_ids=0, ids=None, out=None) == smfg.OK
    assert call("smfg_layer_norm", NORM, max_rows=0, x=None, y=None) == smfg.OK
    assert call("smfg_layer_norm_grad", NGRAD, max_rows=0, x=None, dy=None, mean=None, rstd=None, dw=None, db=None, scratch=None) == smfg.OK


def grads(**change):
    g = smfg._Grad(P, P + 4096, 100, F16, F32, None, 0)
    for k, v in change.items():
        setattr(g, k, v)
    return (smfg._Grad * 1)(g)


def clip(c, n=1, scale=1.0, max_norm=1.0, norm=P, scratch=P & ~255, nbytes=1 << 40):
    return smfg.lib().smfg_clip_grad_norm(c, n, scale, max_norm, norm, scratch, nbytes, None)


def test_clip_refusals():
    size = smfg.lib().smfg_clip_grad_norm_scratch_bytes
    assert size(grads(), 1) > 0 and size(grads(), 0) > 0 and size(None, 0) > 0
    for bad in (dict(numel=-1), dict(numel=1 << 48), dict(dtype=3), dict(out_dtype=BF16), dict(dtype=F32, out_dtype=F16), dict(grad=P + 1), dict(out=P + 2),
                dict(out=P), dict(d_rows=P, row_elems=0), dict(d_rows=P + 4, row_elems=2)):
        assert clip(grads(**bad)) == ARG, bad
        assert size(grads(**bad), 1) == -1, bad
    assert clip(grads(), n=-1) == ARG and size(grads(), -1) == -1 and size(None, 1) == -1
    assert clip(None) == NULL and clip(grads(), norm=None) == NULL and clip(grads(), scratch=None) == NULL and clip(grads(grad=None)) == NULL
    for bad in (dict(scale=float("inf")), dict(scale=float("nan")), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(norm=P + 2),
                dict(scratch=P + 16)):
        assert clip(grads(), **bad) == ARG, bad
    assert clip(grads(), nbytes=200) == ROOM


def test_scratch_sizes_are_host_only():
    L = smfg.lib()
    assert L.smfg_embedding_grad_scratch_bytes(0, 1, 1) >= 0
    for n, rows, dim in ((1, 1, 1), (100_000, 1 << 20, 128), ((1 << 31) - 1, (1 << 31) - 1, 4)):
        assert L.smfg_embedding_grad_scratch_bytes(n, rows, dim) >= 16 * n
    for n, rows, dim in ((-1, 1, 1), (1 << 31, 1, 1), (1, 0, 1), (1, 1 << 31, 1), (1, 1, 0), (1, 1, (1 << 23) + 1)):
        assert L.smfg_embedding_grad_scratch_bytes(n, rows, dim) == -1
        with pytest.raises(smfg.SmfgError):
            smfg.embedding_grad_workspace(n, rows, dim)
    assert L.smfg_layer_norm_grad_scratch_bytes(10, 100) >= 800 and L.smfg_layer_norm_grad_scratch_bytes(0, 100) >= 0
    for n, dim in ((-1, 1), (1 << 31, 1), (1, 0), (1, (1 << 23) + 1)):
        assert L.smfg_layer_norm_grad_scratch_bytes(n, dim) == -1


def test_scratch_has_room_for_calls_of_fewer_ids():
    """Also where a smaller call sorts in other tiles, or in another way."""
    size = smfg.lib().smfg_embedding_grad_scratch_bytes
    for dim in (1, 64, 65, 128, 129, 4096):
        most = 0
        for n in sorted({b + d for b in (0, 256, 2048, 8192, 100_000, 1 << 19, 600_000, 1 << 20, 3_000_000) for d in range(-3, 4) if b + d >= 0}):
            assert size(n, 1000, dim) >= most, (n, dim)
            most = size(n, 1000, dim)


def test_grad_struct_layout_matches_the_binding(tmp_path):
    fields = ["grad", "out", "numel", "dtype", "out_dtype", "d_rows", "row_elems"]
    src = tmp_path / "layout.c"
    src.write_text('#include "smfg.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {\n  printf("size %zu\\n", sizeof(smfg_grad_t));\n'
                   + "\n".join(f'  printf("{f} %zu\\n", offsetof(smfg_grad_t, {f}));' for f in fields) + "\n  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = dict(line.split() for line in subprocess.check_output([str(exe)], text=True).splitlines())
    assert int(got["size"]) == ctypes.sizeof(smfg._Grad)
    for f in fields:
        assert int(got[f]) == getattr(smfg._Grad, f).offset, f
