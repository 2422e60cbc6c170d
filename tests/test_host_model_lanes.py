"""Kernels at a model's two ends on the CPU: their own source, compiled over stand-ins for the device's headers, with the wavefronts
of a workgroup run one at a time between barriers, in several orders.  What hangs on a barrier that is missing comes out wrong
in one of them, where a GPU's wavefronts may run abreast for years."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2512_03644_amd", "csrc")
NATIVE = os.path.join(ROOT, "tests", "native")
CLANG = "/opt/rocm/llvm/bin/clang++"  # (the vector types of the kernels are clang's)


def _run(check, tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("needs clang++")
    here = tmp_path / "csrc"
    here.mkdir()
    # beside the sources, so that they include the stand-in in place of the header
    for f in ("embed.hip", "embed.hpp", "norm.hip", "norm.hpp", "rows.h", "xcd_order.h"):
        shutil.copy(os.path.join(CSRC, f), here)
    shutil.copy(os.path.join(NATIVE, "lanes", "fold.h"), here)
    exe = str(tmp_path / check)
    subprocess.run([CLANG, "-std=c++17", "-O1", "-w", "-ffp-contract=off", "-mf16c", "-I", os.path.join(NATIVE, "lanes"), "-I", str(here), "-I", CSRC,
                    os.path.join(NATIVE, check + ".cpp"), "-o", exe], check=True, capture_output=True, text=True)
    run = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, run.stdout + run.stderr
    assert run.stdout.strip().endswith("ok")


def test_gradients_of_an_embedding_in_any_order_of_wavefronts(tmp_path):
    _run("embed_order_check", tmp_path)


def test_layer_norms_in_any_order_of_wavefronts_and_rows_of_one_value(tmp_path):
    _run("norm_order_check", tmp_path)
