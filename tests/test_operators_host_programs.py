"""Host code of the operators around the layer that needs no device: a refusal, and in small programs of their own the bound of the scored
routing's first products (route_bounds_host.cpp) and the choice of a product's kernel (matmul_plan_host.cpp)."""
import os
import subprocess

import pytest

from paper_2512_17073_amd import binding, build

HERE = os.path.dirname(os.path.abspath(__file__))


def _run(tmp_path, source):
    obj, exe = str(tmp_path / "program.o"), str(tmp_path / "program")
    subprocess.run([build._hipcc(), "--cuda-host-only", "-std=c++17", "-O1", "-fPIC", "-x", "hip", "-c", source, "-o", obj], check=True)
    subprocess.run(["g++", obj, "-o", exe], check=True)     # (no HIP runtime)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_a_token_norm_is_bounded_from_above(tmp_path):
    _run(tmp_path, os.path.join(HERE, "route_bounds_host.cpp"))


@pytest.mark.parametrize("ld_add,ldo,refused", [(72, 64, True), (64, 72, True), (64, 64, False), (72, 72, False)])
def test_a_product_added_in_place_keeps_its_stride(ld_add, ldo, refused):
    """With rows at other distances a workgroup would read what another has written.  (No call here reaches a device: those that are not
    refused for it lack their scales' alignment.)"""
    lib, at = binding.lib(), 0x10000
    args = (at, 256, at if refused else at + 1, at, 256, at, at, ld_add, at, ldo, 4, 256, 64, at, 1 << 40)
    assert lib.moe_lrc_block_matmul(*args, None) == -1
    assert (b"in place" in lib.moe_lrc_last_error()) == refused


def test_the_kernel_of_a_product(tmp_path):
    _run(tmp_path, os.path.join(HERE, "matmul_plan_host.cpp"))
