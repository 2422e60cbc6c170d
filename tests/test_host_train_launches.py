"""What the calls between loss and step enqueue: the library's host code on a recording stand-in for the HIP runtime."""
import os
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2512_03644_amd", "csrc")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_launches_fit_the_device_and_cover_everything(tmp_path):
    def compile_host(src):
        obj = str(tmp_path / (os.path.splitext(os.path.basename(src))[0] + ".o"))
        subprocess.run(["hipcc", "-std=c++17", "-O1", "-w", "-fPIC", "-I", CSRC, "-x", "hip",
                        "--offload-host-only", "-c", "-o", obj, src], check=True, capture_output=True, text=True)
        return obj

    srcs = [os.path.join(CSRC, s) for s in ("api.hip", "kernels.hip", "blocks.hip", "fused.hip", "grads.hip", "policy.hip",
                                              "train_api.hip", "layout.cpp")]
    srcs.append(os.path.join(ROOT, "tests", "native", "train_launches_check.cpp"))
    with ThreadPoolExecutor(len(srcs)) as ex:
        objs = list(ex.map(compile_host, srcs))
    # the device images that the objects would be registered with are absent
    undefined = subprocess.run(["nm", "--undefined-only"] + objs, check=True, capture_output=True, text=True).stdout
    images = sorted({w for w in undefined.split() if w.startswith("__hip_fatbin")})
    exe = str(tmp_path / "train_launches_check")
    subprocess.run([shutil.which("g++") or "c++", "-o", exe] + objs + ["-Wl,--defsym=%s=0" % i for i in images],
                   check=True, capture_output=True, text=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stdout + run.stderr
    assert run.stdout.strip().endswith("ok")
