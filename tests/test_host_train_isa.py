"""What the compiler makes of the kernels between loss and step, where their speed hangs on it and no result shows it."""
import os
import re
import subprocess

import pytest

from paper_2512_03644_amd import build

LLVM = "/opt/rocm/llvm/bin"
SOURCES = ("fused", "grads", "policy")


@pytest.fixture(scope="module")
def code_objects(tmp_path_factory):
    """The device code in the objects that the library is linked from."""
    if not os.path.isdir(LLVM) or not all(os.path.exists(os.path.join(build.OBJ_DIR, s + ".o")) for s in SOURCES):
        pytest.skip("needs the library's objects and the LLVM tools")
    folder, out = tmp_path_factory.mktemp("train"), {}
    for s in SOURCES:
        bundle, out[s] = str(folder / (s + ".fatbin")), str(folder / (s + ".co"))
        subprocess.run([LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + bundle, os.path.join(build.OBJ_DIR, s + ".o"), str(folder / "unused")],
                       check=True, capture_output=True, text=True)
        subprocess.run([LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--input=" + bundle, "--output=" + out[s],
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True, capture_output=True, text=True)
    return out


@pytest.fixture(scope="module")
def registers(code_objects):
    used = {}
    for co in code_objects.values():
        notes = subprocess.run([LLVM + "/llvm-readelf", "--notes", co], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n\s+- \.a", notes)[1:]:  # a kernel's entry begins with .agpr_count
            fields = dict(re.findall(r"\n\s+\.(name|vgpr_count|private_segment_fixed_size):\s+(\S+)", kernel))
            if len(fields) == 3:
                used[fields["name"]] = {k: int(v) for k, v in fields.items() if k != "name"}
    return used


def _check(registers, pattern, count, most):
    found = {k: v for k, v in registers.items() if re.search(pattern, k)}
    assert len(found) == count, sorted(found)
    for k, v in found.items():
        assert v["vgpr_count"] <= most and v["private_segment_fixed_size"] == 0, (k, v)


def test_clipped_steps_keep_nothing_in_scratch_memory(registers):
    # six wavefronts on a SIMD; the long chained bf16 ones without a tally seven: <F16, CHAINED, N, TALLY>
    _check(registers, r"\d+clipped_kernelILb", 18, 80)
    _check(registers, r"\d+clipped_warm_kernelILb", 12, 80)
    _check(registers, r"\d+clipped_kernelILb0ELb1ELj\d+ELb0EE", 3, 72)


def test_norm_clipping_and_policy_loss_keep_nothing_in_scratch_memory(registers):
    _check(registers, r"grad_(norm|clip)_kernel", 4, 128)
    # <DTYPE, THREADS, K, WAVES, ...>: eight wavefronts on a SIMD, or four
    _check(registers, r"policy_kernelILj\dELi\d+ELi\d+ELi8E", 27, 64)
    _check(registers, r"policy_kernelILj\dELi\d+ELi\d+ELi4E", 9, 128)
    _check(registers, r"policy_(sum|grad)_kernel", 9, 64)


def test_short_clipped_steps_load_through_the_caches(code_objects):
    listing = subprocess.run([LLVM + "/llvm-objdump", "-d", "--mcpu=gfx950", code_objects["fused"]], check=True, capture_output=True, text=True).stdout
    nt, name = {}, None
    for line in listing.splitlines():
        m = re.match(r"[0-9a-f]+ <(\S+)>:", line)
        if m:
            name = m.group(1)
        m = re.match(r"\s+(global|flat|buffer)_load_\w+", line)
        if m and name:
            nt.setdefault(name, []).append(bool(re.search(r"\bnt\b", line)))
    warm = [k for k in nt if "clipped_warm_kernel" in k]
    long = [k for k in nt if re.search(r"\d+clipped_kernelILb", k)]
    assert len(warm) == 12 and len(long) == 18
    for k in warm:
        assert not any(nt[k]), k
    for k in long:
        assert any(nt[k]), k
