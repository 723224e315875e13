"""The tree operators in a process with several devices: their host side, linked
with a made-up CUDA runtime (no GPU is used)."""
import os
import subprocess

from conftest import ROOT


def test_launches_are_prepared_on_their_own_device(tmp_path):
    from paper_2504_18583_gb300 import _build
    _build.build()
    exe = str(tmp_path / "fake_devices")
    objs = [os.path.join(_build.BUILD, n + ".cu.o") for n in ("tree_api", "tree", "qk_rope", "sample", "tree_attention")]
    for i, o in enumerate(objs):  # a library that was built elsewhere came without them
        if not os.path.exists(o):
            objs[i] = str(tmp_path / os.path.basename(o))
            subprocess.run([_build.nvcc(), *_build.ARCH, *_build.NVCC_FLAGS, "-c",
                            os.path.join(_build.CSRC, os.path.basename(o)[:-2]), "-o", objs[i]], check=True)
    cuda = os.path.dirname(os.path.dirname(_build.nvcc()))
    subprocess.run(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(cuda, "include"),
                    os.path.join(ROOT, "tests", "fake_devices.cpp"), *objs, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout.strip() == "right", r.stdout + r.stderr
