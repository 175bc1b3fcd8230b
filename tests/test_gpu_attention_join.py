"""A call whose kernel gave up on a wait must not hand out what an older call left in the workspace.  (No test makes such a wait run
out; the kernel that joins the pieces is run alone, on a workspace made by hand.)"""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2609_03079_b200 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("join") / "join.so")
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "join_harness.cu")
    res = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-I", build.CSRC, "-I", os.path.join(build.ROOT, "include"), src, "-o", so], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    L = C.CDLL(so)
    L.run_join.argtypes = [C.c_int] + [C.c_void_p] * 8 + [C.c_int]
    return L


@pytest.mark.parametrize("few_rows", [1, 0])
@pytest.mark.parametrize("ctas,at", [(148, 0), (148, 147), (148, 129), (5, 4), (132, 77)])
def test_rows_of_a_call_that_gave_up_are_nan(harness, few_rows, ctas, at):
    dev = "cuda:0"
    part_o = torch.zeros(4, 64, device=dev)
    part_o[0] = torch.arange(64, device=dev)
    part_lse = torch.zeros(4, device=dev)
    ids = torch.zeros(64 + 5, dtype=torch.int32, device=dev)
    flags = ids[:64].view(torch.uint8)
    seq_len, table, status = (torch.tensor([v], dtype=torch.int32, device=dev) for v in (3, 0, 0))

    def join():
        out = torch.full((64,), -7.0, dtype=torch.bfloat16, device=dev)
        lse = torch.full((1,), -7.0, device=dev)
        torch.cuda.synchronize()
        assert harness.run_join(few_rows, *(t.data_ptr() for t in (out, lse, part_o, part_lse, ids, seq_len, table, status)), ctas) == 0
        return out, lse

    out, lse = join()
    assert torch.equal(out.float(), part_o[0]) and lse.item() == 0
    flags[at] = 1
    out, lse = join()
    assert out.isnan().all() and lse.isnan().all()
    flags[at] = 0
    out, lse = join()
    assert torch.equal(out.float(), part_o[0]) and status.item() == 0
