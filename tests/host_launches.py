"""What the library launches, recorded on the host: the calls of the CUDA runtime that a launch makes are answered by a stand-in, so
that no GPU is needed and nothing runs.  Device pointers are made up.

    Recorder(library).record(calls) -> for every call of the C ABI: (result, [(grid x, threads of a CTA)])

The calls are made in a process of their own, which loads the stand-in ahead of the library and does not import torch (whose
runtime library would be found first)."""
import json
import os
import shutil
import subprocess
import sys
import tempfile

STAND_IN = r"""
#include <cuda_runtime.h>
#include <vector>
namespace { std::vector<long long> seen; }
extern "C" {
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void**)
{
    seen.push_back(c->gridDim.x);
    seen.push_back(c->blockDim.x);
    return cudaSuccess;
}
cudaError_t cudaLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, cudaStream_t)
{
    seen.push_back(grid.x);
    seen.push_back(block.x);
    return cudaSuccess;
}
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
int launches_taken(long long* to, int room)
{
    int n = 0;
    for (; n < (int)seen.size() && n < room; ++n) to[n] = seen[n];
    seen.clear();
    return n;
}
}
"""

CALLER = r"""
import ctypes, json, sys
stand_in = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
T = {"p": ctypes.c_void_p, "i": ctypes.c_int, "l": ctypes.c_int64, "f": ctypes.c_float, "z": ctypes.c_size_t}
room = (ctypes.c_longlong * 64)()
for name, result, types, args in json.load(sys.stdin):
    f = getattr(lib, name)
    f.restype = T[result]
    f.argtypes = [T[t] for t in types]
    got = f(*args)
    n = stand_in.launches_taken(room, 64)
    print(json.dumps([got, [[room[i], room[i + 1]] for i in range(0, n, 2)]]))
"""


class Recorder:
    def __init__(self, library):
        self.library = library
        self.dir = tempfile.mkdtemp(prefix="launches_")
        src, self.so = os.path.join(self.dir, "stand_in.cpp"), os.path.join(self.dir, "stand_in.so")
        with open(src, "w") as f:
            f.write(STAND_IN)
        include = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")
        subprocess.check_call(["g++", "-O1", "-fPIC", "-shared", "-I" + include, src, "-o", self.so])

    def record(self, calls):
        """calls: [(name, result type, types, arguments)] -> [(result, [(grid x, threads)])]"""
        p = subprocess.run([sys.executable, "-c", CALLER, self.so, self.library], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
        assert p.returncode == 0, p.stderr
        return [(got, [tuple(x) for x in launches]) for got, launches in map(json.loads, p.stdout.splitlines())]

    def close(self):
        shutil.rmtree(self.dir, ignore_errors=True)
