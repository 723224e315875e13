"""The bounded wait of the tree attention's warps, compiled from the kernel's own
header: a barrier that nothing completes, an abort, an arrival."""
import ctypes
import os
import subprocess

import pytest
import torch

from conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2504_18583_gb300 import _build
    out = str(tmp_path_factory.mktemp("wait") / "warp_wait.so")
    subprocess.run([_build.nvcc(), *_build.ARCH, *_build.NVCC_FLAGS, "-I" + _build.CSRC, "-shared", "-o", out,
                    os.path.join(ROOT, "tests", "warp_wait.cu")], check=True)
    return ctypes.CDLL(out)


@pytest.mark.parametrize("which,answer,least,most", [(0, 0, 2.0, 2.5), (1, 0, 0.0, 1.0), (2, 1, 0.0, 1.0)])
def test_a_wait_ends(lib, which, answer, least, most):
    """A wait that nothing ends gives up after 2 s and no sooner (the limit that the header documents); one whose
    CTA gives up, or whose barrier completes, ends at once.  All lanes get one answer."""
    answers = torch.full((32,), -1, dtype=torch.int32, device="cuda")
    ns = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert lib.warp_wait_case(which, ctypes.c_void_p(answers.data_ptr()), ctypes.c_void_p(ns.data_ptr())) == 0
    assert answers.tolist() == [answer] * 32
    assert least <= int(ns) * 1e-9 <= most, int(ns)
