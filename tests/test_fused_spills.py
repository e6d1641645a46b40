"""Registers that the kernels with a fused epilogue and the norm keep in scratch
memory, from the metadata of the built library. No GPU."""
import re

from test_gemm_spills import spills  # noqa: F401  (the fixture)


def test_fused_and_gated_kernels_spill_nothing(spills):  # noqa: F811
    # template arguments of the large tiles: 5 + output type (0 to 3), tile height / 64
    mine = {n: s for n, s in spills.items() if re.search(r"2qg5(fused|gated)\d+k_", n)}
    tiles = [n for n in mine if re.search(r"k_gemm_\w+_directILi[5-8]ELi[234]E", n)]
    assert len(tiles) == 2 * (5 * 3 * 4 - 3)  # (no NVFP4 output for bf16 activations)
    assert not any(mine.values()), {n: s for n, s in mine.items() if s}


def test_norm_kernels_spill_nothing(spills):  # noqa: F811
    mine = {n: s for n, s in spills.items() if "k_rms_norm" in n}
    assert len(mine) > 50 and not any(mine.values()), {n: s for n, s in mine.items() if s}
