"""Registers that the compiler put into scratch memory in the built tiled products: the instances that take large
batches keep their sums and addresses in registers."""

import os
import re

import pytest

from paper_2606_05613_amd.build import BUILD


@pytest.mark.parametrize("unit,limit", [("ffn_bf16", 8), ("ffn_f32", 24)])
def test_tiled_products_of_aligned_rows_hardly_spill(unit, limit):
    asm = os.path.join(BUILD, f"{unit}-hip-amdgcn-amd-amdhsa-gfx950.s")
    if not os.path.exists(asm):
        pytest.skip("library not built")
    kernels = re.findall(r"\.name:\s+(_ZN5bkmoo15ffn_tile_kernel\S+).*?\.vgpr_spill_count:\s+(\d+)", open(asm).read(), re.S)
    aligned = {n: int(s) for n, s in kernels if "Lb1EEEv" in n}
    assert len(aligned) == 18  # six products, three sides
    assert {n: s for n, s in aligned.items() if s > limit} == {}
