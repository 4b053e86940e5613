"""Static checks over the compiled gfx950 code of the experts' kernel and of the big tiles that add adapters, with DMA and LDS reads
that the compiler does not see (CPU only: hipcc cross-compiles to assembly, nothing runs)."""
import re
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2511_19438_amd import build as B
from tests.test_isa_checks import check_pending, check_refills, compile_to_asm, kernels


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


@pytest.fixture(scope="module")
def tile_files():
    with tempfile.TemporaryDirectory() as tmp, ThreadPoolExecutor(max_workers=6) as pool:
        jobs = [[f"-DGPTQ_PREFILL_TILE={t}", "-DGPTQ_PREFILL_ADAPTERS"] for t in B.ADAPTER_TILES]
        yield list(pool.map(lambda d: compile_to_asm("prefill_tile.hip", d, tmp), jobs))


def test_tiles_with_adapters_leave_registers_of_pending_lds_reads_alone(tile_files):
    """What follows the tile's loop does not move its operands' registers about, and m0 stays the DMA's."""
    seen = 0
    for path in tile_files:
        for name, lines in kernels(path, labels=True).items():
            seen += 1
            assert "prefill_pipelined_kernel" in name
            tracked = lambda op, in_asm: in_asm and op.startswith("ds_read")  # noqa: E731
            counted = lambda op: op.startswith("ds_") or op.startswith("s_load") or op.startswith("s_buffer_load")  # noqa: E731
            assert not check_pending(lines, tracked, counted, re.compile(r"lgkmcnt\((\d+)\)"), name)
            in_asm = False
            for t in lines:
                in_asm = t.startswith(";;#ASMSTART") or (in_asm and not t.startswith(";;#ASMEND"))
                assert in_asm or not re.search(r"\bm0\b", t), f"{name}: {t}"
    assert seen == 4 * len(B.ADAPTER_TILES) + 2  # (slices one after the other on 64x128)


def test_tiles_with_adapters_spill_nothing(tile_files):
    test_nothing_is_spilled(tile_files)
