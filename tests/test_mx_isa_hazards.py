"""What the assembler does not do for inline assembly, checked in the 4-bit product's device code: see test_isa_hazards.py,
whose checks these are."""
import os
import shutil
import subprocess

import pytest

import test_isa_hazards as isa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    """The device code of mx4.hip as a list of instructions, with the labels of functions and blocks."""
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("isa") / "mx4.s"
    subprocess.run(["hipcc", "-O3", "--offload-arch=gfx950", "-std=c++17", "-ffp-contract=off", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-S", "--cuda-device-only", "-o", str(out), os.path.join(ROOT, "paper_1706_09453_amd", "csrc", "mx4.hip")],
                   check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    lines = [l.split(";")[0].strip() for l in out.read_text().splitlines()]
    return [l for l in lines if l and not l.startswith("//") and (l.endswith(":") or not l.startswith("."))]


def test_no_lds_read_is_under_way_at_a_barrier_of_the_loads_that_write_lds(code):
    isa.test_no_lds_read_is_under_way_at_a_barrier_of_the_loads_that_write_lds(code)


def test_loads_that_write_lds_do_not_read_fresh_sgprs(code):
    isa.test_loads_that_write_lds_do_not_read_fresh_sgprs(code)


def test_product_loops_wait_for_lds_once_a_stage(code):
    """The blocks of a stage's second half are requested between the products of its first half and the other way round: a block with a stage's
    products has one wait for all LDS reads, in front of them (the one at the barrier, which also counts memory, aside; waves of one fragment have no such between)."""
    n, bad = 0, set()
    for name, body in isa._kernels(code):
        if "mx4_gemm_kernel" not in name or "ILi1ELi1E" in name:
            continue
        products, waits = 0, 0
        for ins in body + ["end:"]:
            if ins.endswith(":"):
                n += products > 0
                if products and waits > 1:
                    bad.add(name)
                products = waits = 0
            products += ins.startswith("v_mfma_scale_f32_32x32x64_f8f6f4")
            waits += ins == "s_waitcnt lgkmcnt(0)"
    assert n > 0 and not bad, (n, len(bad), sorted(bad)[:4])
