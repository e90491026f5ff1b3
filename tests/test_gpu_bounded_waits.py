"""Waits of the tensor-core kernel on bounded caches that run out are visible in the result: attention rows are NaN, and so are the masses of every
token that the CTA would have written; nothing hangs, and the device is usable afterwards.  The kernel is compiled here once more, from the same source, with
waits whose number of polls the test sets: none at all in every thread, or none in the second of the two softmax threads of each row alone."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2405_03917_b200 as cq
from paper_2405_03917_b200 import build
from tests import bounded as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
SCALE = 128 ** -0.5

WRAPPER = """
#include <cuda_runtime.h>
__device__ int polls_of[2];                             // softmax threads of the rows' second halves, all others
#define CQ_PREFILL_POLLS polls_of[(threadIdx.x >> 8) == 1 ? 0 : 1]
#include "cq_chunk_attn.cu"
cudaError_t cq::ensure_dynamic_smem(const void* func, int bytes, int)
{
    return cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}
int cq::device_sm_count() { return 148; }
extern "C" {
int set_polls(int second, int others)
{
    const int polls[2] = {second, others};
    return cudaMemcpyToSymbol(polls_of, polls, sizeof polls);
}
// out: attention (fp16) or, with mass not null, masses
int waits_run_out(const void* q, const void* kc, const void* vc, const void* kcb, const void* vcb, const int* lens, float scale, int n_seq, int n_q, int hq,
                  int hkv, int c, long long cap, void* out, float* mass, void* workspace, size_t bytes, void* stream)
{
    cq::BoundedArgs a{};
    cq::Shape& sh = a.sh;
    sh.n_seq = n_seq; sh.max_tokens = cap; sh.n_blocks = (cap + cq::kTokenBlock - 1) / cq::kTokenBlock;
    sh.n_q_heads = hq; sh.n_kv_heads = hkv; sh.head_dim = 128; sh.c = c; sh.b = 8;
    sh.G = 128 / c; sh.K = 256; sh.R = hq / hkv; sh.hb = 0; sh.block_bytes = sh.G * 16;
    a.q = (const __half*)q; a.kc = (const uint8_t*)kc; a.vc = (const uint8_t*)vc; a.kcb = (const __half*)kcb; a.vcb = (const __half*)vcb;
    a.seq_lens = lens; a.n_pages = n_seq; a.pages_per_seq = 1; a.page_blocks = (int)sh.n_blocks; a.n_rows = n_seq * n_q; a.max_q = n_q;
    a.scale_log2e = scale * cq::kLog2e; a.out = (__half*)out; a.most_rows = 1 << 30;
    if (!cq::chunk_attn_supported(sh)) return -1;
    if (!mass) return bytes < cq::chunk_attn_workspace_bytes(a) ? -2 : cq::launch_chunk_attn(a, workspace, bytes, (cudaStream_t)stream);
    return bytes < cq::chunk_mass_workspace_bytes(a) ? -2 : cq::launch_chunk_mass(a, mass, mass, workspace, (cudaStream_t)stream);
}
}
"""


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    nvcc = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc on this machine")
    d = tmp_path_factory.mktemp("bounded")
    src, so = d / "waits.cu", d / "waits.so"
    src.write_text(WRAPPER)
    subprocess.check_call([nvcc, *build.NVCC_FLAGS, "-I" + build.CSRC, "-shared", "-Xlinker", "-Bsymbolic", "-o", str(so), str(src)])
    return ctypes.CDLL(str(so))


class Run:
    def __init__(self, library, c, n_q, hq, hkv, lens):
        self.library, self.n_q, self.cap = library, n_q, max(lens)
        self.case = B.Case(c + n_q, c, 8, hq, hkv, lens, self.cap)
        self.q = self.case.queries(len(lens), n_q)
        self.k, self.v = self.case.contiguous()
        self.lens = self.case.seq_lens()
        self.workspace = torch.zeros(32 << 20, dtype=torch.uint8, device=DEV)

    def __call__(self, polls, out=None, mass=None):
        case, ptr = self.case, lambda t: ctypes.c_void_p(None if t is None else t.data_ptr())
        assert self.library.set_polls(*polls) == 0
        st = self.library.waits_run_out(ptr(self.q), ptr(self.k), ptr(self.v), ptr(case.kcb), ptr(case.vcb), ptr(self.lens), ctypes.c_float(SCALE), case.n, self.n_q,
                                        case.Hq, case.Hkv, case.c, ctypes.c_longlong(self.cap), ptr(out), ptr(mass), ptr(self.workspace),
                                        ctypes.c_size_t(self.workspace.numel()), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0
        torch.cuda.synchronize()
        return out if mass is None else mass


NONE, SECOND, PLENTY = (0, 0), (0, 1 << 17), (1 << 17, 1 << 17)
# one row tile, contexts in several parts; a context in one part; several row tiles; a tile that fills half of a CTA's rows
SHAPES = [(8, 40, 8, 2, [300, 47]), (4, 20, 2, 2, [64]), (2, 300, 4, 4, [500, 310]), (8, 9, 64, 32, [2000, 900, 30])]


@pytest.mark.parametrize("polls", [NONE, SECOND])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_rows_are_nan(library, shape, polls):
    run = Run(library, *shape)
    want = run(PLENTY, torch.zeros_like(run.q))
    assert torch.isfinite(want).all()
    assert torch.isnan(run(polls, torch.zeros_like(run.q))).all()
    assert torch.equal(run(PLENTY, torch.zeros_like(run.q)), want)
    case = run.case
    assert torch.equal(cq.cq_window_attn(run.q, run.k, run.v, case.kcb, case.vcb, run.lens, SCALE, case.c, 8, run.cap, 0, variant=3), want)


@pytest.mark.parametrize("polls", [NONE, SECOND])
@pytest.mark.parametrize("shape", SHAPES)
def test_masses_are_nan(library, shape, polls):
    run = Run(library, *shape)
    case, fresh = run.case, lambda: torch.full((run.case.n, run.case.Hkv, run.cap), 0.25, device=DEV)
    want = run(PLENTY, mass=fresh())
    assert torch.isfinite(want).all()
    run.workspace.zero_()                                                   # what lies there could be taken for sums
    got = run(polls, mass=fresh())
    for s, n in enumerate(case.lens):
        assert torch.isnan(got[s, :, :n]).all(), f"seq {s}: {int((~torch.isnan(got[s, :, :n])).sum())} masses of {n} tokens can be taken for results"
        assert (got[s, :, n:] == 0.25).all()
    assert torch.equal(run(PLENTY, mass=fresh()), want)
