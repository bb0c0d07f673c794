"""The gfx950 code of attention over an 8-bit cache: every instantiation is among the kernels whose loads to LDS are looked at for their wait states (those take their base from
vector registers through v_readfirstlane, which needs five), with ordinary and with nontemporal loads.  Nothing runs on a GPU."""
import os
import re

import pytest

from test_device_code import OBJDUMP
from test_device_code_lds_loads import kernels  # noqa: F401

pytestmark = pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs ROCm's llvm-objdump")


def test_all_instantiations_are_looked_at(kernels):  # noqa: F811
    found = {}
    for name, code in kernels.items():
        m = re.match(r"_ZN5specv24verify_attn_quant_kernelILi(\d)ELi(\d)ELb([01])E", name)
        if m:
            found[m.groups()] = [t for _, t, _ in code]
    assert sorted(found) == [(tiles, type_, ranges) for tiles in "123" for type_ in "01" for ranges in "01"]
    for key, code in found.items():
        loads = [t for t in code if "_load_lds_" in t]
        assert any(t.endswith(" nt") for t in loads) and any(not t.endswith(" nt") for t in loads), key
        assert all(re.search(r"global_load_lds_dwordx4 v\d+, s\[\d+:\d+\]", t) for t in loads), key
        assert any(t.startswith("v_readfirstlane_b32") for t in code), key
