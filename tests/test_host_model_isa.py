"""What the compiler makes of the kernels at a model's two ends, where their speed hangs on it and no result shows it."""
import os
import re
import subprocess

import pytest

from paper_2512_03644_amd import build

LLVM = "/opt/rocm/llvm/bin"
SOURCES = ("embed", "norm", "head")


@pytest.fixture(scope="module")
def code_objects(tmp_path_factory):
    """The device code in the objects that the library is linked from."""
    if not os.path.isdir(LLVM) or not all(os.path.exists(os.path.join(build.OBJ_DIR, s + ".o")) for s in SOURCES):
        pytest.skip("needs the library's objects and the LLVM tools")
    folder, out = tmp_path_factory.mktemp("model"), {}
    for s in SOURCES:
        bundle, out[s] = str(folder / (s + ".fatbin")), str(folder / (s + ".co"))
        subprocess.run([LLVM + "/llvm-objcopy", "--dump-section", ".hip_fatbin=" + bundle, os.path.join(build.OBJ_DIR, s + ".o"), str(folder / "unused")],
                       check=True, capture_output=True, text=True)
        subprocess.run([LLVM + "/clang-offload-bundler", "--unbundle", "--type=o", "--input=" + bundle, "--output=" + out[s],
                        "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"], check=True, capture_output=True, text=True)
    return out


@pytest.fixture(scope="module")
def kernels(code_objects):
    found = {}
    for co in code_objects.values():
        notes = subprocess.run([LLVM + "/llvm-readelf", "--notes", co], check=True, capture_output=True, text=True).stdout
        for kernel in re.split(r"\n\s+- \.a", notes)[1:]:  # a kernel's entry begins with .agpr_count
            fields = dict(re.findall(r"\n\s+\.(name|vgpr_count|private_segment_fixed_size|group_segment_fixed_size):\s+(\S+)", kernel))
            if len(fields) == 4:
                found[fields["name"]] = {k: int(v) for k, v in fields.items() if k != "name"}
    return found


def test_nothing_is_kept_in_scratch_memory(kernels):
    assert len(kernels) > 60
    assert not {k: v for k, v in kernels.items() if v["private_segment_fixed_size"]}


def test_products_leave_room_for_two_wavefronts_on_a_simd_and_their_tiles_in_lds(kernels):
    found = {k: v for k, v in kernels.items() if re.search(r"head_(logits|grads)_kernel", k)}
    assert len(found) == 18
    for k, v in found.items():
        assert v["vgpr_count"] <= 256 and v["group_segment_fixed_size"] <= 160 * 1024, (k, v)
        if re.search(r"logits_kernelILb\dELi64E", k):  # two workgroups on a compute unit
            assert v["vgpr_count"] <= 128 and v["group_segment_fixed_size"] <= 88 * 1024, (k, v)


def test_products_wait_for_loads_at_the_meeting_alone(code_objects):
    """A wait for all loads between a step's reads of LDS and its products would undo the buffers."""
    listing = subprocess.run([LLVM + "/llvm-objdump", "-d", "--mcpu=gfx950", code_objects["head"]], check=True, capture_output=True, text=True).stdout
    for body in re.split(r"\n[0-9a-f]+ <", listing)[1:]:
        if not re.match(r"\S*head_(logits|grads)_kernel", body):
            continue
        lines = body.splitlines()
        loads = [i for i, l in enumerate(lines) if "global_load_lds_dwordx4" in l]
        products = [i for i, l in enumerate(lines) if "v_mfma" in l]
        assert loads and products
        for a, b in zip(products, products[1:]):
            between = [l for l in lines[a + 1:b]]
            if any("s_barrier" in l for l in between) or b - a > 12:
                continue
            assert not any(re.search(r"s_waitcnt .*vmcnt\(0\)", l) for l in between), between
