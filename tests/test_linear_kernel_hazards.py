"""CPU check of the linear-attention kernels' gfx950 assembly: inline assembly holds
no instruction at all (its empty statements only pin values), every transposing
read of LDS comes from the builtin, whose waits the compiler places, and no
kernel spills."""
import os
import re

import pytest

from tests import test_kernel_hazards as rules


@pytest.fixture(scope="module")
def lines(tmp_path_factory):
    if not os.path.exists(rules.HIPCC):
        pytest.skip("hipcc not available")
    path = rules._asm("mtn_linear.hip", str(tmp_path_factory.mktemp("asm")))
    return open(path).read().splitlines()


def test_inline_assembly_is_empty(lines):
    ins = [i for i in rules._instructions(lines) if i]
    assert not [i for i in ins if i[2]]
    assert any(i[0].startswith("ds_read_b64_tr_b16") for i in ins)
    assert any(i[0].startswith("v_mfma_f32_16x16x32") for i in ins)


def test_no_spills(lines):
    spills = [int(m.group(1)) for m in map(re.compile(r"\.vgpr_spill_count:\s+(\d+)").search, lines) if m]
    assert spills and not any(spills)
    assert not [i for i in rules._instructions(lines) if i and i[0].startswith("scratch_")]


def test_no_packed_fp32_arithmetic(lines):
    bad = [i for i in rules._instructions(lines) if i and re.match(r"v_pk_(add|mul|fma)_f32", i[0])]
    assert not bad
