"""Static checks over the compiled gfx950 code of the experts' kernel, whose LDS slots are refilled by DMA that the compiler does
not see (CPU only: hipcc cross-compiles to assembly, nothing runs)."""
import re
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2511_19438_amd import build as B
from tests.test_isa_checks import check_refills, compile_to_asm, kernels


@pytest.fixture(scope="module")
def asm_files():
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(max_workers=6) as pool:
        jobs = [[f"-DGPTQ_EXPERTS_SCALING={s}", f"-DGPTQ_EXPERTS_DOWN={d}"] for s in B.EXPERTS_SCALINGS for d in (0, 1)]
        yield list(pool.map(lambda d: compile_to_asm("experts_scale.hip", d, tmp), jobs))


def instances(asm_files):
    for path in asm_files:
        for name, lines in kernels(path, labels=True).items():
            if "experts_kernel" in name:
                yield name, lines


def test_a_slot_is_refilled_only_after_its_reads(asm_files):
    seen = 0
    for name, lines in instances(asm_files):
        seen += 1
        assert sum(t.startswith("global_load_lds") for t in lines) >= 6 and sum(t.startswith("ds_read") for t in lines) >= 8
        assert check_refills(lines, name) == []
    # four shapes of gate and up and two of down, three numbers of rows, three kinds of group sizes
    assert seen == (4 + 2) * 3 * 3


def test_m0_is_the_dma_s_alone(asm_files):
    for name, lines in instances(asm_files):
        in_asm = False
        for t in lines:
            in_asm = t.startswith(";;#ASMSTART") or (in_asm and not t.startswith(";;#ASMEND"))
            assert in_asm or not re.search(r"\bm0\b", t), f"{name}: {t}"


def test_nothing_is_spilled(asm_files):
    """Two wavefronts to a SIMD: 256 registers each at most."""
    for path in asm_files:
        for entry in re.findall(r"^  - \.agpr_count:.*?(?=^  - |^amdhsa)", open(path).read(), re.S | re.M):
            field = lambda name: int(re.search(rf"\.{name}:\s+(\d+)", entry).group(1))  # noqa: E731
            assert field("vgpr_count") <= 256 and field("vgpr_spill_count") == 0 and field("private_segment_fixed_size") == 0, entry
