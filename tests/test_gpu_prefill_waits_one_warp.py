"""Waits of the tensor-core prefill kernel that run out in one softmax warp alone: that warp goes on without waiting, so what the other warps read may
be the wrong tile's.  No row of such a CTA may come out as a number that is not the result."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2405_03917_b200 as cq
from paper_2405_03917_b200 import build
from tests.test_gpu_prefill_waits import WRAPPER

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def one_warp(tmp_path_factory):
    nvcc = os.environ.get("NVCC") or shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc on this machine")
    d = tmp_path_factory.mktemp("prefill")
    src, so = d / "one_warp.cu", d / "one_warp.so"
    src.write_text(WRAPPER)
    subprocess.check_call([nvcc, *build.NVCC_FLAGS, "-DCQ_PREFILL_POLLS=(threadIdx.x<32?0:1<<17)", "-I" + build.CSRC, "-shared", "-Xlinker", "-Bsymbolic", "-o", str(so),
                           str(src)])
    return ctypes.CDLL(str(so)).prefill_no_polls


@pytest.mark.parametrize("c,n_q,hq,hkv,lens", [(8, 64, 8, 2, [700, 1017]), (4, 3, 2, 2, [64]), (2, 130, 4, 4, [500, 130]), (8, 256, 1, 1, [4000])])
def test_no_row_passes_for_a_result(one_warp, c, n_q, hq, hkv, lens):
    D, n, cap = 128, len(lens), max(lens)
    g = torch.Generator().manual_seed(c)
    q = torch.randn(n, n_q, hq, D, generator=g).half().cuda()
    cb = torch.randn(hkv, D // c, 256, c, generator=g).cuda()
    codes = torch.randint(0, 256, (cq.cq_codes_bytes(n, cap, hkv, D, c, 8),), generator=g, dtype=torch.uint8).cuda()
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = cq.cq_prefill_attn(q, codes, codes, cb, cb, sl, 0.1, c, 8, cap)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    for _ in range(5):
        out = torch.zeros_like(want)
        st = one_warp(ptr(q), ptr(codes), ptr(codes), ptr(cb), ptr(cb), ptr(sl), ctypes.c_float(0.1), n, n_q, hq, hkv, c, ctypes.c_longlong(cap), ptr(out),
                      ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert st == 0
        torch.cuda.synchronize()
        spoilt = torch.isnan(out).all(-1)
        assert spoilt.any()
        wrong = ~spoilt & (out != want).any(-1)
        assert not wrong.any(), f"{int(wrong.sum())} of {wrong.numel()} rows are numbers, but not the result"
    assert torch.equal(cq.cq_prefill_attn(q, codes, codes, cb, cb, sl, 0.1, c, 8, cap), want)
