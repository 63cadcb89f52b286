"""The launches of root-mean-square norm, cross entropy and AdamW, seen on the host: their sources are compiled together with a recorder in the place of the
runtime's launch call, which also refuses what the runtime refuses.  Nothing runs; the addresses are never used."""
import ctypes
import os
import subprocess

import pytest

from paper_2110_08450_amd import binding as smfg
from paper_2110_08450_amd import build

RECORDER = r"""
#include <map>
#include <string>
#include <vector>
#include "rms_norm.hip"
#include "loss.hip"
#include "adamw.hip"
namespace {
struct Launch {
  dim3 blocks, threads;
  const void* kernel;
  uint32_t first;
};
std::vector<Launch> seen;
int fails = -1;  // the launch that fails
hipError_t last = hipSuccess;
std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> m;
  return m;
}
uint32_t first_block(const std::string& name, const void* args) {
  const auto has = [&](const char* s) { return name.find(s) != std::string::npos; };
  if (has("k_rms_norm_grad_long")) return static_cast<const RmsGradArgs*>(args)->first_block;
  if (has("k_rms_norm_long")) return static_cast<const RmsArgs*>(args)->first_block;
  if (has("k_adamw_values")) return static_cast<const AdamValuesArgs*>(args)->first_block;
  if (has("k_adamw")) return static_cast<const AdamArgs*>(args)->first_block;
  return 0;
}
}  // namespace
extern "C" {
void __hipRegisterFunction(void**, const void* kernel, char*, const char* name, unsigned, void*, void*, dim3*, dim3*, int*) { names()[kernel] = name; }
hipError_t hipLaunchKernel(const void* kernel, dim3 blocks, dim3 threads, void** args, size_t, hipStream_t) {
  const bool fits = blocks.x > 0 && blocks.y > 0 && uint64_t(blocks.x) * threads.x < (uint64_t(1) << 32) && blocks.y <= 65535;
  const hipError_t e = fits && static_cast<int>(seen.size()) != fails ? hipSuccess : hipErrorInvalidConfiguration;
  seen.push_back({blocks, threads, kernel, first_block(names()[kernel], args[0])});
  if (e != hipSuccess) last = e;
  return e;
}
hipError_t hipGetLastError() {
  const hipError_t e = last;
  last = hipSuccess;
  return e;
}
void record(int fail) {
  seen.clear();
  fails = fail;
  last = hipSuccess;
}
int count() { return static_cast<int>(seen.size()); }
const char* launch(int i, int64_t* shape) {
  shape[0] = seen[i].blocks.x;
  shape[1] = seen[i].blocks.y;
  shape[2] = seen[i].threads.x;
  shape[3] = seen[i].first;
  return names()[seen[i].kernel].c_str();
}
}
"""
P = 0x7f0000001000  # never dereferenced
F32, F16, BF16, E4M3 = 0, 1, 2, 4
ROOM = 1 << 60
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def rec(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    src, lib = d / "rec.hip", d / "rec.so"
    src.write_text(RECORDER)
    subprocess.run([build.hipcc(), "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-Wno-everything",
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-I", os.path.dirname(build.SRC), "-I", build.INCLUDE, str(src), "-o", str(lib)],
                   check=True, capture_output=True, timeout=600)
    r = ctypes.CDLL(str(lib))
    own = smfg.lib()
    for name in smfg.EXPORTS:
        if name.split("_")[1] in ("rms", "cross", "adamw"):
            f = getattr(r, name)
            f.argtypes, f.restype = getattr(own, name).argtypes, getattr(own, name).restype
    r.launch.restype = ctypes.c_char_p
    return r


def launches(rec):
    """(kernel, blocks, blocks of the second dimension, threads, first block) of the call's launches."""
    out = []
    for i in range(rec.count()):
        shape = (ctypes.c_int64 * 4)()
        name = rec.launch(i, shape).decode()
        out.append((name, *shape))
    return out


def rms(rec, n=1000, dim=100, dtype=F16, ytype=None, group=0):
    return rec.smfg_rms_norm(P, dim, dtype, P + 4096, dim, P + 8192, dim, P, n, dim, P, F32, 1e-5, P + 12288, dim, dtype if ytype is None else ytype,
                             None if ytype is None else P, 1 if group == 0 else -(-dim // group), group, P, None)


def rms_grad(rec, n=1000, dim=100, dtype=F16):
    return rec.smfg_rms_norm_grad(P, dim, P, dim, dtype, P, dim, P, n, dim, P, F32, P, P, dim, P, P, ROOM, None)


def loss(rec, n=1000, classes=172, dtype=F16, mean=True):
    return rec.smfg_cross_entropy(P, classes, dtype, P, 8, P, n, classes, 0 if mean else 1, 1.0, P, P, P, classes, P, ROOM, None)


def adamw(rec, tensors=3, numel=100_000, bits=32, row_elems=0):
    one = smfg._Param(P, P, P, P, P, P, None, numel, F32, F16, 0, bits, 0.1, row_elems, None, None, 0)
    return rec.smfg_adamw((smfg._Param * tensors)(*[one] * tensors), tensors, smfg._AdamW(1e-3, 0.9, 0.999, 1e-8, 1.0, 1.0, 1, None, None, None), None)


def both(rec, tensors=100):
    """States of floats and of 8 bits in turn."""
    ps = [smfg._Param(P, P, P, P, P, P, None, 5000 + i, F32, F16, 0, 32 if i % 2 else 8, 0.1, 0, None, None, 0) for i in range(tensors)]
    return rec.smfg_adamw((smfg._Param * tensors)(*ps), tensors, smfg._AdamW(1e-3, 0.9, 0.999, 1e-8, 1.0, 1.0, 1, None, None, None), None)


def values(rec, numel=100_000, row_elems=0, otype=F32):
    return rec.smfg_adamw_values(P, P, numel, row_elems, 0, P, otype, None)


CALLS = [(rms, {}), (rms, dict(ytype=E4M3, group=32)), (rms, dict(dim=50_000)), (rms, dict(dim=50_000, ytype=E4M3)), (rms_grad, {}), (rms_grad, dict(dim=50_000)),
         (loss, {}), (loss, dict(n=20_000)), (loss, dict(n=20_000, mean=False)), (loss, dict(classes=100_000)), (loss, dict(n=0)), (adamw, {}),
         (adamw, dict(tensors=300, numel=20_000)), (adamw, dict(bits=8)), (both, {}), (adamw, dict(row_elems=100)), (values, {}), (values, dict(row_elems=50))]


@pytest.mark.parametrize("call,sizes", CALLS)
def test_nothing_is_launched_behind_a_launch_that_failed(rec, call, sizes):
    rec.record(-1)
    assert call(rec, **sizes) == smfg.OK
    all_of_them = launches(rec)
    assert all_of_them and all(name for name, *_ in all_of_them)
    for k in range(len(all_of_them)):
        rec.record(k)
        assert call(rec, **sizes) == smfg.ERR_HIP_BASE - 9  # hipErrorInvalidConfiguration
        assert launches(rec) == all_of_them[:k + 1]
        assert rec.hipGetLastError() == 0  # the call has told it


def blocks_of(rec, kernel):
    """Blocks of all launches of the kernel, which have to be one piece behind the other."""
    at = 0
    for name, blocks, _, _, first in launches(rec):
        if kernel in name:
            assert first == at
            at += blocks
    return at


def ceil(a, b):
    return -(-a // b)


@pytest.mark.parametrize("n,dim,dtype", [(1, 50_000, F16), (2 ** 24 + 1, 8193, F32), (MOST, 16_385, BF16), (MOST, 1 << 23, F32), (MOST, 64, F16), (MOST, 4096, F32)])
def test_norm_of_up_to_2_31_rows(rec, n, dim, dtype):
    for call, kernel in ((rms, "k_rms_norm_long"), (rms_grad, "k_rms_norm_grad_long"), (lambda *a, **k: rms(*a, ytype=E4M3, **k), "k_rms_norm_long")):
        rec.record(-1)
        assert call(rec, n=n, dim=dim, dtype=dtype) == smfg.OK
        assert blocks_of(rec, kernel) == (n if dim > 8192 else 0)


@pytest.mark.parametrize("n", [1, 8192, 8193, MOST])
@pytest.mark.parametrize("classes", [1, 7, 172, 4096, 57_344, 57_345, 1 << 23])
@pytest.mark.parametrize("dtype", [F32, F16])
def test_loss_of_up_to_2_31_rows(rec, n, classes, dtype):
    """One launch over the rows, one for the loss where several blocks have them, and one for the labels where there are many."""
    rec.record(-1)
    assert loss(rec, n=n, classes=classes, dtype=dtype) == smfg.OK
    names = [name for name, *_ in launches(rec)]
    assert len(names) == (3 if n > 8192 else 2 if n > 1 else 1) and ("k_loss_count" in names[0]) == (n > 8192) and ("k_loss_join" in names[-1]) == (n > 1)
    assert ("k_cross_entropy_long" in names[-2 if n > 1 else 0]) == (classes > (57_344 if dtype == F16 else 28_672))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_many_and_large_tensors(rec, bits):
    """36 tensors to a launch; blocks of 1024 elements, or more where there would be over a million of them."""
    for tensors in (1, 36, 37, 290):
        rec.record(-1)
        assert adamw(rec, tensors=tensors, numel=10_000, bits=bits) == smfg.OK
        assert rec.count() == ceil(tensors, 36)
    for numel, each in ((1, 1024), (2 ** 30, 1024), (2 ** 31, 2048), (2 ** 45, 65_536)):
        rec.record(-1)
        each = max(each, 2048) if bits == 8 else each
        assert adamw(rec, tensors=1, numel=numel, bits=bits) == smfg.OK
        assert blocks_of(rec, "k_adamw") == ceil(numel, each)
    rec.record(-1)
    assert adamw(rec, tensors=1, numel=2 ** 48 - 1, bits=bits) == smfg.ERR_INVALID_ARG and rec.count() == 0
    rec.record(-1)
    assert both(rec, 100) == smfg.OK and rec.count() == 4


def test_values_of_large_states(rec):
    for numel in (1, 8192, 8193, 2 ** 40):
        rec.record(-1)
        assert values(rec, numel=numel) == smfg.OK
        assert blocks_of(rec, "k_adamw_values") == ceil(numel, 8192)
    rec.record(-1)
    assert values(rec, numel=2 ** 48 - 1) == smfg.ERR_INVALID_ARG and rec.count() == 0
