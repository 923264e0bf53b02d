"""The adapter calls' host code with a recorder in the place of the HIP runtime: which kernels a call launches, in which grids, and which parts of the
workspace they are given, without a GPU.  The library's own sources are compiled for the host alone; no kernel exists in the result."""
import collections
import ctypes
import os
import subprocess

import pytest

from paper_2605_26660_amd import binding, build

RECORDER = r"""
#include <cstdlib>
#include <map>
#include <string>
#include <vector>
#include "windq_adapters.hpp"
using namespace windq;

struct Launch { std::string name; uint64_t grid, block; };
struct Region { uint64_t from, to; };
static std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
static std::vector<Launch> launches;
static std::vector<Region> regions;                        // of the workspace, that the recorded launches write side by side
static dim3 grid_, block_;

static void shrink_part(const ShrinkArgs& S) {
    const uint64_t at = reinterpret_cast<uint64_t>(S.part);
    regions.push_back({at, at + (uint64_t)S.slots * S.splits * GROUP * shrink_ranks(S.A.max_rank) * 4});
}
static void join_planes(const JoinArgs& J) {
    const uint64_t at = reinterpret_cast<uint64_t>(J.planes);
    if (J.planes != nullptr) regions.push_back({at, at + (uint64_t)J.slots * GROUP * J.A.max_rank * 6});
}

extern "C" {
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* host, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[host] = name; }
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t, hipStream_t) { grid_ = g; block_ = b; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* g, dim3* b, size_t* s, hipStream_t* st) { *g = grid_; *b = block_; *s = 0; *st = nullptr; return hipSuccess; }
hipError_t hipLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t, hipStream_t) {
    const std::string name = names()[f];
    launches.push_back({name, (uint64_t)g.x * g.y * g.z, (uint64_t)b.x * b.y * b.z});
    if (name.find("shrink_kernel") != std::string::npos || name.find("join_kernelENS_8JoinArgs") != std::string::npos) {
        const int64_t first2 = *static_cast<int64_t*>(args[2]);
        const bool two = (int64_t)g.x > first2;
        if (name.find("shrink_kernel") != std::string::npos) {
            shrink_part(*static_cast<ShrinkArgs*>(args[0]));
            if (two) shrink_part(*static_cast<ShrinkArgs*>(args[1]));
        } else {
            join_planes(*static_cast<JoinArgs*>(args[0]));
            if (two) join_planes(*static_cast<JoinArgs*>(args[1]));
        }
    }
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipPeekAtLastError() { return hipSuccess; }

void recorded_nothing() { std::abort(); }
void recorded_clear() { launches.clear(); regions.clear(); }
int64_t recorded_launches() { return (int64_t)launches.size(); }
const char* recorded_name(int64_t i) { return launches[i].name.c_str(); }
uint64_t recorded_grid(int64_t i) { return launches[i].grid; }
uint64_t recorded_block(int64_t i) { return launches[i].block; }
int64_t recorded_regions() { return (int64_t)regions.size(); }
uint64_t recorded_region(int64_t i, int32_t end) { return end != 0 ? regions[i].to : regions[i].from; }
}
"""

Launch = collections.namedtuple("Launch", "name grid block")
AT = 1 << 40                                     # an address on every alignment, never read


class Recorder:
    def __init__(self, path):
        self.lib = ctypes.CDLL(path)
        binding._declare(self.lib, ctypes.POINTER)
        i64, u64 = ctypes.c_int64, ctypes.c_uint64
        for name, args, res in (("launches", [], i64), ("name", [i64], ctypes.c_char_p), ("grid", [i64], u64), ("block", [i64], u64), ("regions", [], i64),
                                ("region", [i64, ctypes.c_int32], u64), ("clear", [], None)):
            f = getattr(self.lib, "recorded_" + name)
            f.argtypes, f.restype = args, res

    def launches(self):
        L = self.lib
        return [Launch(L.recorded_name(i).decode(), L.recorded_grid(i), L.recorded_block(i)) for i in range(L.recorded_launches())]

    def regions(self):
        L = self.lib
        return [(L.recorded_region(i, 0), L.recorded_region(i, 1)) for i in range(L.recorded_regions())]

    def product(self, grad, T, rows, cols, G=128, unit_rows=0, dtype=binding.WINDQ_BF16, n=0, rank=0, mask=False, w_dtype=None, ld_dy=None, h=False, want_dx=True,
                codes_bytes=1 << 40, packed=True, side=True):
        """One call of windq_project (grad: windq_project_grad) with made-up addresses. -> (status, workspace's address, its bytes)"""
        B, L = binding, self.lib
        W = B.windq_mat(AT, dtype if w_dtype is None else w_dtype, 0, rows, cols, cols)
        X = B.windq_mat(AT, dtype, 0, T, cols, cols)
        dY = B.windq_mat(AT, dtype, 0, T, rows, rows if ld_dy is None else ld_dy)
        P = B.windq_packed(ctypes.pointer(W), AT if mask else None, AT, AT, AT, codes_bytes, AT, AT, G, 0, unit_rows)
        A = B.windq_adapters(AT, AT, AT, AT, n, rank, dtype, 0)
        ref = ctypes.byref
        need = L.windq_project_workspace_bytes(int(grad), dtype, T, rows, cols, G, n, rank)
        L.recorded_clear()
        p, a = ref(P) if packed else None, ref(A) if n else None
        if grad:
            side = AT if n and side else None
            status = L.windq_project_grad(p, ref(dY), ref(X) if n else None, a, AT, AT if h else None, AT if want_dx else None, cols, side, side, AT, need, None)
        else:
            status = L.windq_project(p, ref(X), a, AT, AT, rows, AT if h else None, AT, need, None)
        return status, AT, need


@pytest.fixture(scope="session")
def recorder(tmp_path_factory):
    try:
        hipcc = build.hipcc_path()
    except RuntimeError:
        pytest.skip("no hipcc")
    at = tmp_path_factory.mktemp("recorder")
    (at / "recorder.hip").write_text(RECORDER)
    sources = [str(at / "recorder.hip")] + [os.path.join(build.CSRC, s) for s in build.SOURCES]
    flags = ["--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-fPIC", "-w", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC]
    objs = [str(at / (os.path.basename(s) + ".o")) for s in sources]
    jobs = [subprocess.Popen([hipcc, *flags, "-c", s, "-o", o], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for s, o in zip(sources, objs)]
    for j in jobs:
        out = j.communicate()[0]
        assert j.returncode == 0, out
    path = str(at / "librecorder.so")
    # the rest of the runtime, and the symbols that would hold the kernels' code: nobody calls or reads them
    symbols = lambda which, files: set(subprocess.run(["nm", "-j", which, *files], check=True, capture_output=True, text=True).stdout.split())
    missing = sorted(s for s in symbols("-u", objs) - symbols("--defined-only", objs) if s.startswith(("hip", "__hip")))
    held = ["-Wl,--defsym=%s=%s" % (s, "0" if s.startswith("__hip_fatbin") else "recorded_nothing") for s in missing]
    subprocess.run(["g++", "-shared", "-Wl,-Bsymbolic", *held, *objs, "-o", path], check=True, capture_output=True)
    return Recorder(path)
