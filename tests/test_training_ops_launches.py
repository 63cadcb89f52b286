"""The launches of the training operators, seen on the host: their source is compiled together with a recorder in the place of the
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
#include "train.hip"
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
// The first block of a launch, where its arguments say one.
template <typename A>
auto first_of(const void* args, int) -> decltype(static_cast<const A*>(args)->first_block) {
  return static_cast<const A*>(args)->first_block;
}
template <typename A>
uint32_t first_of(const void*, long) {
  return 0;
}
uint32_t first_block(const std::string& name, const void* args) {
  const auto has = [&](const char* s) { return name.find(s) != std::string::npos; };
  if (has("k_embedding")) return first_of<EmbedArgs>(args, 0);
  if (has("k_embed_sums")) return first_of<EmbedGradArgs>(args, 0);
  if (has("k_layer_norm_long")) return first_of<NormArgs>(args, 0);
  if (has("k_layer_norm_grad_long")) return first_of<NormGradArgs>(args, 0);
  if (has("k_clip_squares") || has("k_clip_scale")) return first_of<ClipArgs>(args, 0);
  return 0;
}
}  // namespace
extern "C" {
void __hipRegisterFunction(void**, const void* kernel, char*, const char* name, unsigned, void*, void*, dim3*, dim3*, int*) { names()[kernel] = name; }
// a launch written kernel<<<blocks, threads>>>(...) puts its shape here
dim3 shape[2];
hipError_t __hipPushCallConfiguration(dim3 blocks, dim3 threads, size_t, hipStream_t) {
  shape[0] = blocks;
  shape[1] = threads;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* blocks, dim3* threads, size_t* lds, hipStream_t* stream) {
  *blocks = shape[0];
  *threads = shape[1];
  *lds = 0;
  *stream = nullptr;
  return hipSuccess;
}
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
int clip_many(int64_t tensors, int64_t numel) {
  std::vector<smfg_grad_t> g(tensors, smfg_grad_t{reinterpret_cast<void*>(0x7f0000001000), nullptr, numel, SMFG_DTYPE_F32, 0, nullptr, 0});
  return smfg_clip_grad_norm(g.data(), static_cast<int32_t>(tensors), 1.f, 1.f, reinterpret_cast<float*>(0x7f0000001000), reinterpret_cast<void*>(0x7f0000001000),
                             int64_t(1) << 60, nullptr);
}
}
"""
P = 0x7f0000001000  # never dereferenced
F32, F16, BF16 = 0, 1, 2
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
        if name.split("_")[1] in ("embedding", "layer", "clip"):
            f = getattr(r, name)
            f.argtypes, f.restype = getattr(own, name).argtypes, getattr(own, name).restype
    r.launch.restype = ctypes.c_char_p
    r.clip_many.argtypes = [ctypes.c_int64, ctypes.c_int64]
    return r


def launches(rec):
    """(kernel, blocks, blocks of the second dimension, threads, first block) of the call's launches."""
    out = []
    for i in range(rec.count()):
        shape = (ctypes.c_int64 * 4)()
        name = rec.launch(i, shape).decode()
        out.append((name, *shape))
    return out


def embedding(rec, n=1000, rows=5000, dim=100, table=F16, out=F16):
    return rec.smfg_embedding(P, rows, dim, table, P, 8, P, n, dim, 1.0, P, dim, out, None)


def grad(rec, n=1000, rows=5000, dim=100, dy=F16, grad=F32, accumulate=0):
    return rec.smfg_embedding_grad(P, 4, P, n, P, dim, dy, dim, 1.0, P, rows, dim, grad, accumulate, P, ROOM, None)


def grad_rows(rec, n=1000, rows=5000, dim=100, dy=F16, grad=F32):
    return rec.smfg_embedding_grad_rows(P, 4, P, n, P, dim, dy, dim, 1.0, rows, P, P, P, dim, grad, P, ROOM, None)


def norm(rec, n=1000, dim=100, dtype=F16):
    return rec.smfg_layer_norm(P, dim, dtype, P, n, dim, P, P, F32, 1e-5, P, dim, P, P, None)


def norm_grad(rec, n=1000, dim=100, dtype=F16):
    return rec.smfg_layer_norm_grad(P, dim, P, dim, dtype, P, n, dim, P, F32, P, P, P, dim, P, P, P, ROOM, None)


def clip(rec, tensors=3, numel=100_000):
    return rec.clip_many(tensors, numel)


CALLS = [(embedding, {}), (grad, dict(n=100)), (grad, {}), (grad, dict(n=30_000)), (grad, dict(n=1_200_000, accumulate=1)), (grad, dict(n=0)),
         (grad_rows, dict(n=9)), (grad_rows, dict(n=2000)), (grad_rows, dict(n=20_000, rows=1 << 20)), (grad_rows, dict(n=3_000_000)), (grad_rows, dict(n=0)),
         (norm, {}), (norm, dict(dim=50_000)), (norm_grad, {}), (norm_grad, dict(dim=50_000)), (clip, {}), (clip, dict(tensors=300, numel=20_000))]


@pytest.mark.parametrize("call,sizes", CALLS)
def test_nothing_is_launched_behind_a_launch_that_failed(rec, call, sizes):
    """Later launches work on what earlier ones leave in the scratch."""
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


@pytest.mark.parametrize("n", [1, 1000, 2 ** 30 - 1, 2 ** 30 + 1, MOST])
@pytest.mark.parametrize("dim,dy,columns", [(1, F16, 1), (64, F16, 1), (128, BF16, 2), (8200, F32, 4)])
def test_gradient_of_up_to_2_31_ids(rec, n, dim, dy, columns):
    """Every launch has fewer work items than 2^32, and together they have the blocks of all tokens."""
    tiles = ceil(ceil(dim, columns), 64)
    # few rows: cleared by blocks of the same launches, a row or more each
    for call, sizes, clearing in ((grad, dict(rows=2, accumulate=1), 0), (grad, dict(rows=2), ceil(2, max(1, min(512, 32768 // (dim * 4))))),
                                  (grad_rows, dict(rows=1000), 0)):
        rec.record(-1)
        assert call(rec, n=n, dim=dim, dy=dy, **sizes) == smfg.OK
        assert blocks_of(rec, "k_embed_sums") == (ceil(n, 128) if n > 256 else 1) * tiles + clearing


@pytest.mark.parametrize("n", [0, 1, 256, 257, 30_000, 2 ** 30])
@pytest.mark.parametrize("dim,dtype,bytes_", [(1, F16, 2), (32, F16, 2), (20, F32, 4), (5000, F32, 4), (12_000, BF16, 2)])
def test_gradient_of_a_table_of_up_to_2_31_rows(rec, n, dim, dtype, bytes_):
    """The blocks that clear are as many as they have to be, in launches that the runtime takes; or the sort's clear everything."""
    rec.record(-1)
    assert grad(rec, n=n, rows=MOST, dim=dim, dy=dtype, grad=dtype) == smfg.OK
    names = [name for name, *_ in launches(rec)]
    if n > 256 and MOST >= 2 * n:
        assert any("k_sort" in name for name in names)
    else:
        rows = max(1, min(512, 32768 // (dim * bytes_)))
        columns = 1 if dim <= 64 else 2 if dim <= 128 else 4
        assert blocks_of(rec, "k_embed_sums") == (ceil(n, 128) if n > 256 else min(n, 1)) * ceil(ceil(dim, columns), 64) + ceil(MOST, rows)


@pytest.mark.parametrize("n,dim,out,vector", [(1, 1, F16, 8), (MOST, 1, F32, 4), (MOST, 7, F16, 8), (MOST, 65, F16, 8), (MOST, 1024, F32, 4), (1000, 1 << 23, F32, 4)])
def test_lookup_of_up_to_2_31_ids(rec, n, dim, out, vector):
    rec.record(-1)
    assert embedding(rec, n=n, dim=dim, table=out, out=out) == smfg.OK
    assert blocks_of(rec, "k_embedding") == ceil(n * ceil(dim, vector if dim >= vector else 1), 1024)


@pytest.mark.parametrize("n,dim,dtype", [(1, 50_000, F16), (2 ** 24 + 1, 8193, F32), (MOST, 16_385, BF16), (MOST, 1 << 23, F32), (MOST, 64, F16), (MOST, 4096, F32)])
def test_norm_of_up_to_2_31_rows(rec, n, dim, dtype):
    for call, kernel in ((norm, "k_layer_norm_long"), (norm_grad, "k_layer_norm_grad_long")):
        rec.record(-1)
        assert call(rec, n=n, dim=dim, dtype=dtype) == smfg.OK
        assert blocks_of(rec, kernel) == (n if dim > 8192 else 0)


def test_clipping_of_up_to_2_31_blocks(rec):
    for tensors, numel in ((1, 1), (1, (1 << 48) - 1), (5, 1 << 42), (20_000_000, 3)):
        rec.record(-1)
        # two thousand elements to a block, or as many more as leave 4096 blocks, at most 2^16
        chunk = 2048
        while chunk < 65536 and tensors * numel > 8192 * chunk:
            chunk *= 2
        blocks = tensors * ceil(numel, chunk)
        if blocks >= 2 ** 31:
            assert clip(rec, tensors, numel) == smfg.ERR_INVALID_ARG and rec.count() == 0
            continue
        assert clip(rec, tensors, numel) == smfg.OK
        assert blocks_of(rec, "k_clip_squares") == blocks == blocks_of(rec, "k_clip_scale")


def test_more_blocks_than_have_numbers_are_refused_before_anything_is_launched(rec):
    rec.record(-1)
    assert embedding(rec, n=MOST, dim=1 << 23) == smfg.ERR_INVALID_ARG
    assert grad(rec, n=MOST, dim=1 << 23) == smfg.ERR_INVALID_ARG
    assert grad_rows(rec, n=MOST, dim=1 << 23) == smfg.ERR_INVALID_ARG
    assert rec.smfg_embedding_grad_scratch_bytes(MOST, 1000, 1 << 23) == -1
    assert rec.count() == 0
