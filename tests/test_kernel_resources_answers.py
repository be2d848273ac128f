"""The kernels of 8-bit products and of log-probabilities as they are built: none of the epilogues keeps its accumulators in memory, and the
row kernels, which have a wave per SIMD for each 64 registers, none of their row."""
import re

import pytest

from test_kernel_resources import code_objects, readelf  # noqa: F401 (a fixture)


@pytest.fixture(scope="module")
def use(code_objects):  # noqa: F811
    """kernel name -> (vector registers, spilled ones, bytes of scratch)"""
    found = {}
    for path in code_objects:
        for kernel in readelf("--notes", path).split("  - .agpr_count:")[1:]:
            field = dict(re.findall(r"^    \.(\w+): +(\S+)$", kernel, re.M))
            found[field["name"]] = tuple(int(field[k]) for k in ("vgpr_count", "vgpr_spill_count", "private_segment_fixed_size"))
    return found


@pytest.mark.parametrize("parameters,tiles,spilled", [("GemmIntParams", 12, 0), ("GemmStatsParams", 13, 5), ("GemmIntStatsParams", 12, 22)])
def test_gemm_kinds(use, parameters, tiles, spilled):
    """The 256 x 256 tile of the statistics spills what its epilogue holds of scales and sums beside 256 accumulators, the others nothing."""
    kinds = {n: v for n, v in use.items() if re.search(r"gemm_mi16_kernel.*\d%sE" % parameters, n)}
    assert len(kinds) == 2 * tiles
    for name, (_, spills, scratch) in kinds.items():
        full = "ILi8ELi8E" in name
        assert spills <= (spilled if full else 0) and scratch <= (4 * spilled + 16 if full else 0), (name, spills, scratch)


def test_row_kernels(use):
    rows = {n: v for n, v in use.items() if re.search(r"logprob_(rows|pieces)_kernel|quantise_rows_kernel|few_rows_kernel|some_rows_kernel", n)}
    assert len(rows) == 16 + 2 + 3 + 6 + 8
    for name, (registers, spills, scratch) in rows.items():
        assert spills == 0 and scratch == 0, (name, spills, scratch)
        if "logprob_rows" in name:
            assert registers <= 64, (name, registers)
