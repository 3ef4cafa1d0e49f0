"""CPU check of the int8 kernels' gfx950 assembly: the rules of
test_kernel_hazards (inline assembly, M0 and permlane wait states, no spills in
loops that stream through LDS DMA) on their source."""
import os

import pytest

from tests import test_kernel_hazards as rules


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not os.path.exists(rules.HIPCC):
        pytest.skip("hipcc not available")
    path = rules._asm("mtn_i8.hip", str(tmp_path_factory.mktemp("asm")))
    return {"mtn_i8.hip": open(path).read().splitlines()}


@pytest.mark.parametrize("rule", ["test_no_vector_alu_instruction_in_inline_asm",
                                  "test_lds_dma_asm_waits_after_its_m0_write",
                                  "test_permlane_swaps_are_compiler_placed_with_wait_states",
                                  "test_no_spill_traffic_inside_dma_loops"])
def test_rule(listings, rule):
    getattr(rules, rule)(listings)
